// Matrix products of the word-model operators (include/lda_ops.h): the gated
// layer and the softmax cross entropy, forward and backward.
//
// Every product is C[m][n] = sum_k L[m][k] R[n][k] with both operands
// contiguous in k, on the matrix units; what is done with C (activation,
// softmax statistics, gradient of the logits, store) is the epilogue of the
// kernel that computes it, while C is still in registers.
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
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ------------------------------------------------------------ tile product --
// One 16-byte fragment of each operand per lane: row lane & 15, 16-byte chunk
// lane >> 4 of 64 bytes of k.  The matrix instruction takes R as its first
// operand, so lane l of the result holds C[m = l & 15][n = 4 (l >> 4) + r],
// r = 0..3: four neighbours along the contiguous axis of C.
template <typename T>
__device__ inline f32x4 mma(u32x4 r, u32x4 l, f32x4 c);
template <>
__device__ inline f32x4 mma<bf16>(u32x4 r, u32x4 l, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r), __builtin_bit_cast(bf16x8, l), c, 0, 0,
                                                 0);
}
template <>
__device__ inline f32x4 mma<f16>(u32x4 r, u32x4 l, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, r), __builtin_bit_cast(f16x8, l), c, 0, 0,
                                                0);
}
// single precision: the four values of a chunk go to four instructions; the
// sum over k does not care that k is dealt out by fours
template <>
__device__ inline f32x4 mma<float>(u32x4 r, u32x4 l, f32x4 c) {
  const f32x4 a = __builtin_bit_cast(f32x4, r), b = __builtin_bit_cast(f32x4, l);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Rows of an operand.  Rows past the end repeat the last one: their products
// go nowhere, and no read leaves the matrix.
template <typename T>
struct Rows {
  const T *p;
  int64_t ld;
  int rows;
  __device__ const char *row(int r) const {
    return reinterpret_cast<const char *>(p + int64_t(min(r, rows - 1)) * ld);
  }
};

// Rows of w_gate and w_value in turns of 16: row n of the pair is row
// (n / 32) * 16 + n % 16 of w_gate where n & 16 is 0, else of w_value.  A lane
// that holds a fragment of a then holds the same elements of b in the next.
__device__ inline int pair_row(int n) { return (n >> 5) * 16 + (n & 15); }
template <typename T>
struct PairRows {
  const T *gate, *value;
  int64_t ld_gate, ld_value;
  int rows;
  __device__ const char *row(int n) const {
    const int64_t f = min(pair_row(n), rows - 1);
    return reinterpret_cast<const char *>(n & 16 ? value + f * ld_value : gate + f * ld_gate);
  }
};

// What the epilogue of a workgroup's wave needs to know.
struct Place {
  int m0, n0;  // first row of L and of R of the wave's part of the tile
  int mt, nt;  // the workgroup's tile
  int wm, wn;  // the wave in the workgroup
  int lane, split;
  char *lds;
};

struct Grid {
  int mtiles, ntiles;
  int chunks;        // 16-byte chunks of k
  int steps, split;  // 128-byte steps of k in all, and of one split
};

// 16 bytes that every lane whose chunk lies past the end of k reads instead
__device__ const u32x4 kZeroChunk = {0, 0, 0, 0};

typedef const __attribute__((address_space(1))) void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;

// Tile order: the tiles are cut into eight runs, one for each accelerator die
// (workgroups go to the dies in turn), and a run walks groups of eight tile
// rows column by column, so that the tiles a die works on at one time share
// their operands in its L2.
__device__ inline bool tile_of(const Grid &g, int &mt, int &nt) {
  const int tiles = g.mtiles * g.ntiles;
  const int per = (tiles + 7) >> 3;
  const int t = int(blockIdx.x & 7) * per + int(blockIdx.x >> 3);
  if (int(blockIdx.x >> 3) >= per || t >= tiles) return false;
  const int group = 8 * g.ntiles, first = t / group * 8;
  const int high = min(8, g.mtiles - first), in = t % group;
  mt = first + in % high;
  nt = in / high;
  return true;
}

// C tile of BM x BN by WM x WN waves.  Each step loads 128 bytes of k of every
// row straight into LDS (two buffers, the next step's loads in flight while
// this step's fragments are multiplied).  A row is eight 16-byte chunks; chunk
// c of row r lies at place c ^ (r & 7), so that the 16 rows that a fragment
// read touches spread over the banks.
template <typename T, int BM, int BN, int WM, int WN, typename L, typename R, typename Epilogue>
__global__ __launch_bounds__(64 * WM *WN) void k_product(Grid g, L left, R right, Epilogue epilogue) {
  constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16, WAVES = WM * WN;
  constexpr int LOADS = (BM + BN) / 8 / WAVES;  // 1 KiB loads of one wave and step
  constexpr int STAGE = (BM + BN) * 128;
  static_assert((BM / 8) % WAVES == 0 && (BN / 8) % WAVES == 0, "a wave's loads are all of one operand's kind");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int mt, nt;
  if (!tile_of(g, mt, nt)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;

  const int chunk = (lane & 7) ^ (lane >> 3);
  const char *src[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (i * WAVES + wave) * 8 + (lane >> 3);
    src[i] = (i * WAVES * 8 < BM ? left.row(mt * BM + r) : right.row(nt * BN + r - BM)) + chunk * 16;
  }
  const int begin = int(blockIdx.z) * g.split, end = min(g.steps, begin + g.split);

  auto load = [&](int step, int stage) {
    char *to = lds + stage * STAGE + wave * 1024;
    if (step * 8 + 8 <= g.chunks) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        __builtin_amdgcn_global_load_lds((global_ptr)(src[i] + int64_t(step) * 128),
                                         (lds_ptr)(to + i * WAVES * 1024), 16, 0, 0);
    } else {
      const bool in = step * 8 + chunk < g.chunks;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const char *p = in ? src[i] + int64_t(step) * 128 : reinterpret_cast<const char *>(&kZeroChunk);
        __builtin_amdgcn_global_load_lds((global_ptr)p, (lds_ptr)(to + i * WAVES * 1024), 16, 0, 0);
      }
    }
  };

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

  if (begin < end) load(begin, 0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int step = begin; step < end; ++step) {
    const int stage = (step - begin) & 1;
    if (step + 1 < end) load(step + 1, stage ^ 1);
    const char *tl = lds + stage * STAGE + wm * TM * 128, *tr = lds + stage * STAGE + (BM + wn * TN) * 128;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int place = (((s * 4 + (lane >> 4)) ^ (lane & 7)) * 16) + (lane & 15) * 128;
      u32x4 fl[MI], fr[NI];
#pragma unroll
      for (int i = 0; i < MI; ++i) fl[i] = *reinterpret_cast<const u32x4 *>(tl + i * 2048 + place);
#pragma unroll
      for (int j = 0; j < NI; ++j) fr[j] = *reinterpret_cast<const u32x4 *>(tr + j * 2048 + place);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mma<T>(fr[j], fl[i], acc[i][j]);
    }
    // the next step's loads have landed, and every wave is done with this one
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  epilogue(Place{mt * BM + wm * TM, nt * BN + wn * TN, mt, nt, wm, wn, lane, int(blockIdx.z), lds}, acc);
}

// ------------------------------------------------------------- epilogues ----
template <typename T>
__device__ inline void store4(T *p, f32x4 v, int count, bool whole) {
  if (whole && count >= 4) {
    typedef T vec __attribute__((ext_vector_type(4)));
    *reinterpret_cast<vec *>(p) = vec{T(v[0]), T(v[1]), T(v[2]), T(v[3])};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < count) p[r] = T(v[r]);
  }
}

template <typename T>
__device__ inline f32x4 load4(const T *p, int count, bool whole) {
  f32x4 v = {0, 0, 0, 0};
  if (whole && count >= 4) {
    typedef T vec __attribute__((ext_vector_type(4)));
    const vec w = *reinterpret_cast<const vec *>(p);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = float(w[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < count) v[r] = float(p[r]);
  }
  return v;
}

// Where row m of a product's result goes: a matrix, or w_gate's and w_value's
// gradients in turns of 16 rows (pair_row).
template <typename T>
struct Target {
  T *p, *q;
  int64_t ld;
  int rows;  // of p (and q)
  bool pair;
  bool whole;           // four columns can be stored at once
  const float *factor;  // of the result, on the device; NULL = 1
  __device__ T *row(int m) const {
    const int f = pair ? pair_row(m) : m;
    if (f >= rows) return nullptr;
    return (pair && (m & 16) ? q : p) + f * ld;
  }
};

template <typename T>
struct Store {
  Target<T> out;
  int cols;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
    const float f = out.factor ? *out.factor : 1.0f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      T *row = out.row(at.m0 + i * 16 + (at.lane & 15));
      if (!row) continue;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = at.n0 + j * 16 + (at.lane >> 4) * 4;
        if (n < cols) store4(row + n, c[i][j] * f, cols - n, out.whole);
      }
    }
  }
};

// One split's part of the result, in 32 bits: [split][rows][cols4], added to
// what an earlier launch left there if `add`.
struct StorePart {
  float *part;
  int rows, cols4;
  bool add;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
      float *row = part + (int64_t(at.split) * rows + m) * cols4;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = at.n0 + j * 16 + (at.lane >> 4) * 4;
        if (n >= cols4) continue;
        f32x4 *p = reinterpret_cast<f32x4 *>(row + n);
        *p = add ? *p + c[i][j] : c[i][j];
      }
    }
  }
};

// The activation and its derivative.
__device__ inline void gate(int act, float a, float &p, float &dp) {
  if (act == LDA_GELU) {
    const float phi = 0.5f * erfcf(-a * 0.70710678118654752f);
    p = a * phi;
    dp = phi + a * 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.5f * kLog2e * a * a);
    return;
  }
  // sigmoid(a) and 1 - sigmoid(a) from e = exp(-|a|), which does not overflow
  const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(a)), big = 1.0f / (1.0f + e), small = e * big;
  const float s = a >= 0.0f ? big : small, t = a >= 0.0f ? small : big;
  if (act == LDA_SIGMOID) {
    p = s;
    dp = s * t;
  } else {
    p = a * s;
    dp = s + a * s * t;
  }
}

template <typename T>
struct GatedForward {
  T *h;
  int64_t ld;
  int rows, hidden, act;
  bool whole;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
#pragma unroll
      for (int j = 0; j < NI; j += 2) {
        const int f = pair_row(at.n0 + j * 16) + (at.lane >> 4) * 4;
        if (f >= hidden) continue;
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p, dp;
          gate(act, c[i][j][r], p, dp);
          v[r] = p * c[i][j + 1][r];
        }
        store4(h + m * ld + f, v, hidden - f, whole);
      }
    }
  }
};

// da and db in turns of 16 columns (pair_row), zero past `hidden`: operands of
// the backward products.
template <typename T>
struct GatedBackward {
  const T *dh;
  int64_t ld;
  T *dab;  // [rows][pair_cols]
  int rows, hidden, pair_cols, act;
  bool whole;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
#pragma unroll
      for (int j = 0; j < NI; j += 2) {
        const int n = at.n0 + j * 16 + (at.lane >> 4) * 4, f = pair_row(n);
        if (n >= pair_cols) continue;
        const f32x4 d = load4(dh + m * ld + f, hidden - f, whole);
        f32x4 da, db;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p, dp;
          gate(act, c[i][j][r], p, dp);
          da[r] = f + r < hidden ? d[r] * c[i][j + 1][r] * dp : 0.0f;
          db[r] = f + r < hidden ? d[r] * p : 0.0f;
        }
        T *out = dab + int64_t(m) * pair_cols + n;
        store4(out, da, 4, true);
        store4(out + 16, db, 4, true);
      }
    }
  }
};

__device__ inline float exp_diff(float z, float top) { return __builtin_amdgcn_exp2f((z - top) * kLog2e); }

// The logits of four words: past the vocabulary -inf.
__device__ inline f32x4 logits(f32x4 c, const float *bias, int v, int vocab) {
#pragma unroll
  for (int r = 0; r < 4; ++r) c[r] = v + r < vocab ? (bias ? c[r] + bias[v + r] : c[r]) : -INFINITY;
  return c;
}

// Per row and tile of words: the largest logit and the sum of exp(z - it), and
// the label's logit from the lane that holds it.
template <int BM, int WN>
struct SoftmaxPart {
  const float *bias;
  const int32_t *labels;
  float *label_logit;  // [rows]
  float2 *part;        // [ntiles][rows]
  int rows, vocab;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
    float2 *shared = reinterpret_cast<float2 *>(at.lds);  // [WN][BM]
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = at.m0 + i * 16 + (at.lane & 15);
      const int label = m < rows ? labels[m] : -1;
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int v = at.n0 + j * 16 + (at.lane >> 4) * 4;
        c[i][j] = logits(c[i][j], bias, v, vocab);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          top = fmaxf(top, c[i][j][r]);
          if (v + r == label && label < vocab) label_logit[m] = c[i][j][r];
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      // nothing but -inf: the sum is 0 against any finite reference
      const float ref = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += exp_diff(c[i][j][r], ref);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (at.lane < 16) shared[at.wn * BM + at.wm * MI * 16 + i * 16 + at.lane] = make_float2(top, sum);
    }
    __syncthreads();
    const int m = at.mt * BM + int(threadIdx.x);
    if (threadIdx.x < BM && m < rows) {
      float2 a = shared[threadIdx.x];
#pragma unroll
      for (int w = 1; w < WN; ++w) {
        const float2 b = shared[w * BM + threadIdx.x];
        const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.0f : top;
        a = make_float2(top, a.y * exp_diff(a.x, ref) + b.y * exp_diff(b.x, ref));
      }
      part[int64_t(at.nt) * rows + m] = a;
    }
  }
};

// G of one piece of the vocabulary (words from `first` on), and its column
// sums by tile of rows.
template <typename T, int BN, int WM>
struct SoftmaxGrad {
  const float *bias;
  const int32_t *labels;
  const float *lse, *dloss, *scale;  // scale[0]: of G's values in type T
  T *grad;                           // [rows][ldg]
  int64_t ldg;
  float *col_part;  // [mtiles][piece], NULL without a bias
  int rows, vocab, first, piece;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
    f32x4 sums[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j) sums[j] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = at.m0 + i * 16 + (at.lane & 15);
      const int label = m < rows ? labels[m] : -1;
      const float l = m < rows ? lse[m] : 0.0f;
      const bool kept = label >= 0 && label < vocab && l != -INFINITY;
      const float d = kept ? dloss[m] * scale[0] : 0.0f;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = at.n0 + j * 16 + (at.lane >> 4) * 4, v = first + n;
        const f32x4 z = logits(c[i][j], bias, v, vocab);
        f32x4 grad;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          grad[r] = kept ? d * (exp_diff(z[r], l) - (v + r == label ? 1.0f : 0.0f)) : 0.0f;
        if (m < rows && n < ldg) store4(grad_row(m) + n, grad, 4, true);
        sums[j] += grad;
      }
    }
    if (!col_part) return;
    float *shared = reinterpret_cast<float *>(at.lds);  // [WM][BN]
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float s = sums[j][r];
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) s += __shfl_xor(s, x);
        if ((at.lane & 15) == 0) shared[at.wm * BN + at.wn * NI * 16 + j * 16 + (at.lane >> 4) * 4 + r] = s;
      }
    __syncthreads();
    const int n = at.nt * BN + int(threadIdx.x);
    if (threadIdx.x < BN && n < piece) {
      float s = shared[threadIdx.x];
#pragma unroll
      for (int w = 1; w < WM; ++w) s += shared[w * BN + threadIdx.x];
      col_part[int64_t(at.mt) * piece + n] = s;
    }
  }
  __device__ T *grad_row(int m) const { return grad + m * ldg; }
};

// ---------------------------------------------------------- small kernels ---
// Joins the parts of a row: 16 rows a workgroup, 16 threads a row.
__global__ __launch_bounds__(256) void k_lse_join(const float2 *part, int ntiles, const float *label_logit,
                                                  const int32_t *labels, int rows, int vocab, float *loss, float *lse) {
  __shared__ float2 shared[16][17];
  const int m = blockIdx.x * 16 + (threadIdx.x & 15), way = threadIdx.x >> 4;
  float2 a = make_float2(-INFINITY, 0.0f);
  if (m < rows)
    for (int t = way; t < ntiles; t += 16) {
      const float2 b = part[int64_t(t) * rows + m];
      const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.0f : top;
      a = make_float2(top, a.y * exp_diff(a.x, ref) + b.y * exp_diff(b.x, ref));
    }
  shared[way][threadIdx.x & 15] = a;
  __syncthreads();
  if (threadIdx.x < 16 && m < rows) {
    for (int w = 1; w < 16; ++w) {
      const float2 b = shared[w][threadIdx.x];
      const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.0f : top;
      a = make_float2(top, a.y * exp_diff(a.x, ref) + b.y * exp_diff(b.x, ref));
    }
    const float total = a.x == -INFINITY && a.y == 0.0f ? -INFINITY : a.x + kLn2 * __builtin_amdgcn_logf(a.y);
    lse[m] = total;
    const int label = labels[m];
    float out = 0.0f;
    if (label >= 0 && label < vocab) {
      const float z = label_logit[m];
      out = z == -INFINITY ? INFINITY : total - z;
    }
    loss[m] = out;
  }
}

// The largest finite |dloss| of the rows kept, as a factor that brings G to
// the range of its type and its inverse: out[0] = unit / top, out[1] = top /
// unit (0 and 0 where no row has a gradient).
__global__ __launch_bounds__(1024) void k_grad_scale(const float *dloss, const int32_t *labels, int rows, int vocab,
                                                     float unit, float *out) {
  __shared__ float shared[16];
  float top = 0.0f;
  for (int m = threadIdx.x; m < rows; m += 1024) {
    const float d = fabsf(dloss[m]);
    if (labels[m] >= 0 && labels[m] < vocab && d < INFINITY) top = fmaxf(top, d);
  }
  for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 16; ++w) top = fmaxf(top, shared[w]);
    // a top below 2^-100 would overflow its inverse: it counts as that
    top = top > 0.0f ? fmaxf(top, 0x1p-100f) : 0.0f;
    out[0] = top > 0.0f ? unit / top : 0.0f;
    out[1] = top / unit;
  }
}

// out[n] = factor * sum over t of part[t][n]
__global__ __launch_bounds__(256) void k_sum_parts(const float *part, int count, int n_all, const float *factor,
                                                   float *out) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= n_all) return;
  float s = 0.0f;
  for (int t = 0; t < count; ++t) s += part[int64_t(t) * n_all + n];
  out[n] = s * *factor;
}

// Joins the splits of a product.
template <typename T>
__global__ __launch_bounds__(256) void k_join(const float *part, int splits, int rows, int cols, int cols4,
                                              Target<T> out) {
  const int64_t all = int64_t(rows) * cols4, step = int64_t(gridDim.x) * 1024;
  for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; at < all; at += step) {
    const int m = int(at / cols4), n = int(at % cols4);
    T *row = out.row(m);
    if (!row || n >= cols) continue;
    f32x4 s = *reinterpret_cast<const f32x4 *>(part + at);
    for (int z = 1; z < splits; ++z) s += *reinterpret_cast<const f32x4 *>(part + z * all + at);
    if (out.factor) s *= *out.factor;
    store4(row + n, s, cols - n, out.whole);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero(T *p, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = T(0.0f);
}

// Copies for the products, zero where the source ends: dst[r][c] = src[r][c],
// or transposed dst[c][r] = src[r][c], in 64 x 64 tiles.
template <typename T>
struct Pack {
  const T *src;
  int64_t ld;
  int rows, cols;
  T *dst;
  int64_t ldd;
  int dst_rows, dst_cols;
  const int32_t *labels;  // rows whose label is outside [0, vocab) are zero; NULL = none
  int vocab;
  int pair;  // transposed only: 0 = dst column r; 1, 2 = the places of w_gate's, w_value's rows among the pair's
};

template <typename T, bool Transposed>
__global__ __launch_bounds__(256) void k_pack(Pack<T> a) {
  __shared__ T tile[64][65];
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  for (int i = threadIdx.x; i < 4096; i += 256) {
    const int r = r0 + (i >> 6), c = c0 + (i & 63);
    T v = T(0.0f);
    if (r < a.rows && c < a.cols) {
      v = a.src[int64_t(r) * a.ld + c];
      if (a.labels && (a.labels[r] < 0 || a.labels[r] >= a.vocab)) v = T(0.0f);
    }
    tile[i >> 6][i & 63] = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 4096; i += 256) {
    const int u = i >> 6, w = i & 63;
    if (Transposed) {
      const int c = c0 + u, r = r0 + w;
      const int at = a.pair ? (r >> 4) * 32 + (r & 15) + (a.pair - 1) * 16 : r;
      if (c < a.dst_rows && at < a.dst_cols) a.dst[int64_t(c) * a.ldd + at] = tile[w][u];
    } else {
      const int r = r0 + u, c = c0 + w;
      if (r < a.dst_rows && c < a.dst_cols) a.dst[int64_t(r) * a.ldd + c] = tile[u][w];
    }
  }
}

// ------------------------------------------------------------------- host ---
constexpr int kTile = 128;

// Workgroups of a kernel that strides over its elements.
unsigned strided(int64_t workgroups) { return unsigned(workgroups < 65536 ? workgroups : 65536); }

#define OPS_TRY(expr)                      \
  do {                                     \
    hipError_t e_ = (expr);                \
    if (e_ != hipSuccess) return e_;       \
  } while (0)

template <typename T>
constexpr int chunk_elems() {
  return 16 / int(sizeof(T));
}

template <typename T>
bool whole4(const void *p, int64_t ld) {
  return reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T)) == 0 && ld % 4 == 0;
}

// Whether an operand can be read where it lies: its rows start at multiples of
// 16 bytes and hold whole chunks.
template <typename T>
bool in_place(const void *p, int64_t ld, int64_t cols) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % chunk_elems<T>() == 0 && cols % chunk_elems<T>() == 0;
}

template <typename T>
hipError_t pack(const Pack<T> &a, bool transposed, hipStream_t s) {
  // the tiles cover the source and the padding of the copy
  const int64_t rows = transposed ? (a.pair ? ceil_div(a.dst_cols, 2) : a.dst_cols) : a.dst_rows;
  const int64_t cols = transposed ? a.dst_rows : a.dst_cols;
  const int64_t most = 65535 * 64;  // of one launch's grid along the rows
  for (int64_t r = 0; r < rows; r += most) {
    Pack<T> b = a;
    if (r) {
      b.src += r * a.ld;
      b.rows = int(a.rows - r);
      b.dst += transposed ? (a.pair ? 2 * r : r) : r * a.ldd;
      if (transposed) b.dst_cols -= int(a.pair ? 2 * r : r);
      else b.dst_rows -= int(r);
      if (a.labels) b.labels += r;
    }
    const dim3 grid(unsigned(ceil_div(cols, 64)), unsigned(ceil_div(rows - r < most ? rows - r : most, 64)));
    if (transposed) k_pack<T, true><<<grid, 256, 0, s>>>(b);
    else k_pack<T, false><<<grid, 256, 0, s>>>(b);
    OPS_TRY(hipGetLastError());
  }
  return hipSuccess;
}

// An operand of a product over its columns, copied where it has to be.
template <typename T>
hipError_t operand(const void *p, int64_t ld, int rows, int cols, Arena &ws, bool dry, hipStream_t s, Rows<T> &out) {
  if (in_place<T>(p, ld, cols)) {
    out = Rows<T>{static_cast<const T *>(p), ld, rows};
    return hipSuccess;
  }
  const int64_t ldd = round_up(cols, chunk_elems<T>());
  T *copy = ws.take<T>(int64_t(rows) * ldd);
  out = Rows<T>{copy, ldd, rows};
  if (dry) return hipSuccess;
  return pack(Pack<T>{static_cast<const T *>(p), ld, rows, cols, copy, ldd, rows, int(ldd), nullptr, 0, 0}, false, s);
}

template <typename T, typename L, typename R, typename Epilogue>
hipError_t product(int64_t m, int64_t n, int64_t k, int splits, const L &left, const R &right, const Epilogue &epi,
                   hipStream_t s) {
  Grid g;
  g.mtiles = int(ceil_div(m, kTile));
  g.ntiles = int(ceil_div(n, kTile));
  g.chunks = int(ceil_div(k, chunk_elems<T>()));
  g.steps = (g.chunks + 7) / 8;
  g.split = int(ceil_div(g.steps, splits));
  const dim3 grid(unsigned(round_up(int64_t(g.mtiles) * g.ntiles, 8)), 1, unsigned(splits));
  auto kernel = k_product<T, kTile, kTile, 2, 2, L, R, Epilogue>;
  const size_t lds = 2 * (kTile + kTile) * 128;
  kernel<<<grid, 256, lds, s>>>(g, left, right, epi);
  return hipGetLastError();
}

// How many ways the sum over k is split: enough workgroups for the device,
// each with at least eight steps.
template <typename T>
int splits_for(int64_t m, int64_t n, int64_t k) {
  const int64_t tiles = ceil_div(m, kTile) * ceil_div(n, kTile);
  const int64_t steps = ceil_div(k, 8 * chunk_elems<T>());
  int64_t want = ceil_div(512, tiles);
  if (want > steps / 8) want = steps / 8;
  return int(want < 1 ? 1 : want > 64 ? 64 : want);
}

// A whole product into `out`, split over k where it has few tiles.
template <typename T, typename L, typename R>
hipError_t product_into(int64_t m, int64_t n, int64_t k, const L &left, const R &right, const Target<T> &out, Arena &ws,
                        bool dry, hipStream_t s) {
  const int splits = splits_for<T>(m, n, k);
  const int64_t cols4 = round_up(n, 4);
  float *part = splits > 1 ? ws.take<float>(splits * m * cols4) : nullptr;
  if (dry) return hipSuccess;
  if (splits == 1) return product<T>(m, n, k, 1, left, right, Store<T>{out, int(n)}, s);
  OPS_TRY(product<T>(m, n, k, splits, left, right, StorePart{part, int(m), int(cols4), false}, s));
  k_join<T><<<strided(ceil_div(m * cols4, 1024)), 256, 0, s>>>(part, splits, int(m), int(n), int(cols4), out);
  return hipGetLastError();
}

template <typename T>
hipError_t zero(T *p, int64_t n, hipStream_t s) {
  k_zero<T><<<strided(ceil_div(n, 256)), 256, 0, s>>>(p, n);
  return hipGetLastError();
}

// The places of w_gate's and w_value's rows among the pair's, padding included.
int64_t pair_cols(int hidden) { return 2 * round_up(hidden, 64); }

template <typename T>
hipError_t pair_operands(const lda_gated_args &a, Arena &ws, bool dry, hipStream_t s, PairRows<T> &out) {
  Rows<T> g, v;
  OPS_TRY(operand<T>(a.w_gate, a.ld_gate, a.hidden, a.width, ws, dry, s, g));
  OPS_TRY(operand<T>(a.w_value, a.ld_value, a.hidden, a.width, ws, dry, s, v));
  out = PairRows<T>{g.p, v.p, g.ld, v.ld, a.hidden};
  return hipSuccess;
}

template <typename T>
hipError_t gated_forward_t(const lda_gated_args &a, Arena &ws, bool dry) {
  if (a.rows == 0) return hipSuccess;
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  Rows<T> x;
  PairRows<T> w;
  OPS_TRY(operand<T>(a.x, a.ldx, int(a.rows), a.width, ws, dry, s, x));
  OPS_TRY(pair_operands<T>(a, ws, dry, s, w));
  if (dry) return hipSuccess;
  const GatedForward<T> epi{static_cast<T *>(a.h), a.ldh, int(a.rows), a.hidden, a.act, whole4<T>(a.h, a.ldh)};
  return product<T>(a.rows, pair_cols(a.hidden), a.width, 1, x, w, epi, s);
}

template <typename T>
hipError_t gated_backward_t(const lda_gated_args &a, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  T *dwg = static_cast<T *>(a.dw_gate), *dwv = static_cast<T *>(a.dw_value);
  if (a.rows == 0) {
    if (dry) return hipSuccess;
    OPS_TRY(zero(dwg, int64_t(a.hidden) * a.width, s));
    return zero(dwv, int64_t(a.hidden) * a.width, s);
  }
  const int rows = int(a.rows), pc = int(pair_cols(a.hidden));
  const int64_t rows_k = round_up(a.rows, chunk_elems<T>());
  Rows<T> x;
  PairRows<T> w;
  OPS_TRY(operand<T>(a.x, a.ldx, rows, a.width, ws, dry, s, x));
  OPS_TRY(pair_operands<T>(a, ws, dry, s, w));
  T *dab = ws.take<T>(a.rows * pc);
  T *dab_t = ws.take<T>(int64_t(pc) * rows_k);
  T *x_t = ws.take<T>(int64_t(a.width) * rows_k);
  T *w_t = ws.take<T>(int64_t(a.width) * pc);
  if (!dry) {
    const GatedBackward<T> epi{static_cast<const T *>(a.dh), a.lddh, dab, rows, a.hidden, pc, a.act,
                               whole4<T>(a.dh, a.lddh)};
    OPS_TRY(product<T>(a.rows, pc, a.width, 1, x, w, epi, s));
    OPS_TRY(pack(Pack<T>{dab, pc, rows, pc, dab_t, rows_k, pc, int(rows_k), nullptr, 0, 0}, true, s));
    OPS_TRY(pack(Pack<T>{static_cast<const T *>(a.x), a.ldx, rows, a.width, x_t, rows_k, a.width, int(rows_k), nullptr,
                         0, 0}, true, s));
    OPS_TRY(pack(Pack<T>{static_cast<const T *>(a.w_gate), a.ld_gate, a.hidden, a.width, w_t, pc, a.width, pc, nullptr,
                         0, 1}, true, s));
    OPS_TRY(pack(Pack<T>{static_cast<const T *>(a.w_value), a.ld_value, a.hidden, a.width, w_t, pc, a.width, pc,
                         nullptr, 0, 2}, true, s));
  }
  const Target<T> dx{static_cast<T *>(a.dx), nullptr, a.lddx, rows, false, whole4<T>(a.dx, a.lddx), nullptr};
  OPS_TRY(product_into<T>(a.rows, a.width, pc, Rows<T>{dab, pc, rows}, Rows<T>{w_t, pc, a.width}, dx, ws, dry, s));
  const Target<T> dw{dwg, dwv, a.width, a.hidden, true, whole4<T>(dwg, a.width) && whole4<T>(dwv, a.width), nullptr};
  return product_into<T>(pc, a.width, a.rows, Rows<T>{dab_t, rows_k, pc}, Rows<T>{x_t, rows_k, a.width}, dw, ws, dry,
                         s);
}

template <typename T>
hipError_t xent_forward_t(const lda_xent_args &a, Arena &ws, bool dry) {
  if (a.rows == 0) return hipSuccess;
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const int rows = int(a.rows), ntiles = int(ceil_div(a.vocab, kTile));
  Rows<T> x, w;
  OPS_TRY(operand<T>(a.x, a.ldx, rows, a.width, ws, dry, s, x));
  OPS_TRY(operand<T>(a.weight, a.ld_weight, a.vocab, a.width, ws, dry, s, w));
  float2 *part = ws.take<float2>(int64_t(ntiles) * rows);
  float *label_logit = ws.take<float>(rows);
  if (dry) return hipSuccess;
  const SoftmaxPart<kTile, 2> epi{a.bias, a.labels, label_logit, part, rows, a.vocab};
  OPS_TRY(product<T>(a.rows, a.vocab, a.width, 1, x, w, epi, s));
  k_lse_join<<<unsigned(ceil_div(rows, 16)), 256, 0, s>>>(part, ntiles, label_logit, a.labels, rows, a.vocab, a.loss,
                                                          a.lse);
  return hipGetLastError();
}

// Words of one piece: G of a piece takes at most 256 MiB.
template <typename T>
int piece_words(int64_t rows, int vocab) {
  const int64_t most = (int64_t(256) << 20) / (rows * int64_t(sizeof(T))) / kTile * kTile;
  const int64_t all = round_up(vocab, kTile);
  return int(most < 1024 ? (all < 1024 ? all : 1024) : most < all ? most : all);
}

template <typename T>
hipError_t xent_backward_t(const lda_xent_args &a, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  T *dw = static_cast<T *>(a.dweight);
  if (a.rows == 0) {
    if (dry) return hipSuccess;
    OPS_TRY(zero(dw, int64_t(a.vocab) * a.width, s));
    return a.dbias ? zero(a.dbias, a.vocab, s) : hipSuccess;
  }
  const int rows = int(a.rows), piece = piece_words<T>(a.rows, a.vocab);
  const int64_t rows_k = round_up(a.rows, chunk_elems<T>());
  const int mtiles = int(ceil_div(a.rows, kTile));
  Rows<T> x, w;
  OPS_TRY(operand<T>(a.x, a.ldx, rows, a.width, ws, dry, s, x));
  OPS_TRY(operand<T>(a.weight, a.ld_weight, a.vocab, a.width, ws, dry, s, w));
  float *scale = ws.take<float>(2);
  T *grad = ws.take<T>(a.rows * piece);
  T *grad_t = ws.take<T>(int64_t(piece) * rows_k);
  T *x_t = ws.take<T>(int64_t(a.width) * rows_k);
  T *w_t = ws.take<T>(int64_t(a.width) * piece);
  float *col_part = a.bias ? ws.take<float>(int64_t(mtiles) * piece) : nullptr;
  const int splits = splits_for<T>(a.rows, a.width, piece);
  const int64_t cols4 = round_up(a.width, 4);
  float *dx_part = ws.take<float>(splits * a.rows * cols4);
  if (!dry) {
    // half precision: G up to 2^14, so that small probabilities are not lost
    // below its smallest normal value
    k_grad_scale<<<1, 1024, 0, s>>>(a.dloss, a.labels, rows, a.vocab, sizeof(T) == 2 ? 16384.0f : 1.0f, scale);
    OPS_TRY(hipGetLastError());
    OPS_TRY(pack(Pack<T>{static_cast<const T *>(a.x), a.ldx, rows, a.width, x_t, rows_k, a.width, int(rows_k),
                         a.labels, a.vocab, 0}, true, s));
  }
  // the pieces' products share the scratch of their parts
  const size_t mark = ws.used;
  size_t most = mark;
  for (int first = 0; first < a.vocab; first += piece) {
    const int words = a.vocab - first < piece ? a.vocab - first : piece;
    const int words_k = int(round_up(words, chunk_elems<T>()));
    const Rows<T> wp{w.p + int64_t(first) * w.ld, w.ld, words};
    ws.used = mark;
    if (!dry) {
      const SoftmaxGrad<T, kTile, 2> epi{a.bias, a.labels, a.lse, a.dloss, scale, grad, words_k, col_part, rows, a.vocab,
                                         first, words};
      OPS_TRY(product<T>(a.rows, words_k, a.width, 1, x, wp, epi, s));
      if (a.dbias) {
        k_sum_parts<<<unsigned(ceil_div(words, 256)), 256, 0, s>>>(col_part, mtiles, words, scale + 1,
                                                                   a.dbias + first);
        OPS_TRY(hipGetLastError());
      }
      OPS_TRY(pack(Pack<T>{grad, words_k, rows, words, grad_t, rows_k, words, int(rows_k), nullptr, 0, 0}, true, s));
      OPS_TRY(pack(Pack<T>{wp.p, wp.ld, words, a.width, w_t, words_k, a.width, words_k, nullptr, 0, 0}, true, s));
      OPS_TRY(product<T>(a.rows, a.width, words_k, splits, Rows<T>{grad, words_k, rows}, Rows<T>{w_t, words_k, a.width},
                         StorePart{dx_part, rows, int(cols4), first > 0}, s));
    }
    T *dwp = dw + int64_t(first) * a.width;
    const Target<T> out{dwp, nullptr, a.width, words, false, whole4<T>(dwp, a.width), scale + 1};
    OPS_TRY(product_into<T>(words, a.width, a.rows, Rows<T>{grad_t, rows_k, words}, Rows<T>{x_t, rows_k, a.width}, out,
                            ws, dry, s));
    if (ws.used > most) most = ws.used;
  }
  ws.used = most;
  if (dry) return hipSuccess;
  const Target<T> out{static_cast<T *>(a.dx), nullptr, a.lddx, rows, false, whole4<T>(a.dx, a.lddx), scale + 1};
  k_join<T><<<strided(ceil_div(a.rows * cols4, 1024)), 256, 0, s>>>(dx_part, splits, rows, a.width, int(cols4), out);
  return hipGetLastError();
}

}  // namespace

#define BY_TYPE(fn, ...)                              \
  switch (a.dtype) {                                  \
    case LDA_F32: return fn<float>(__VA_ARGS__);      \
    case LDA_BF16: return fn<bf16>(__VA_ARGS__);      \
    default: return fn<f16>(__VA_ARGS__);             \
  }

hipError_t gated_forward(const lda_gated_args &a, Arena &ws, bool dry) { BY_TYPE(gated_forward_t, a, ws, dry) }
hipError_t gated_backward(const lda_gated_args &a, Arena &ws, bool dry) { BY_TYPE(gated_backward_t, a, ws, dry) }
hipError_t xent_forward(const lda_xent_args &a, Arena &ws, bool dry) { BY_TYPE(xent_forward_t, a, ws, dry) }
hipError_t xent_backward(const lda_xent_args &a, Arena &ws, bool dry) { BY_TYPE(xent_backward_t, a, ws, dry) }

}  // namespace ops
}  // namespace lda
