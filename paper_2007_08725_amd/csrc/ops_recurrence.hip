// Gated linear recurrence over documents (include/lda_ops.h): forward, backward
// and single steps.
//
// h_t = f_t h_{t-1} + b_t is a chain in each column.  A wave holds kRows rows of
// its columns in registers and reduces them to one map, state in -> state out,
// m -> A m + B; a workgroup joins its waves' maps in LDS, and workgroups, which
// start in the order of the rows, pass the state on through memory: each leaves
// its map, or, as soon as it has it, the state after its last row, looks back
// until it finds a state, and applies the maps between in their order.  So
// every input is read once and every output written once, and the results are
// those of one fixed order of the operations whichever workgroup was faster.
// A document's first row cuts the chain: a map with a first row in it does not
// depend on the state that comes in.
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

constexpr int kRows = LDA_OPS_RECUR_ROWS;  // of a wave
constexpr int kWaves = 8;
constexpr int kBlock = kRows * kWaves;  // rows of a workgroup
constexpr int kAhead = 4;               // maps that a wave looks back to at a time
constexpr int kWindow = kAhead * kWaves;

constexpr float kLog2e = 1.4426950408889634f;

// f = sigmoid(g) and k = 1 - f from e = exp(-g), each to a few roundings of
// itself: e stays below 2^120, so that e f is finite.
template <typename T>
__device__ inline void gate(float g, float &f, float &k) {
  float t = -kLog2e * g;
  t = t > 120.0f ? 120.0f : t;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (sizeof(T) == 4) {
    // what the product with log2 e was rounded by
    const float low = __builtin_fmaf(-kLog2e, g, -t) - 1.9259629911266175e-8f * g;
    if (fabsf(t) < 120.0f) e = __builtin_fmaf(e, 0.6931471805599453f * low, e);
  }
  f = __builtin_amdgcn_rcpf(1.0f + e);
  k = e * f;
}

// N columns of a lane, side by side; N > 1 are moved as 32 bits.
template <typename T, int N>
struct Raw {
  typedef T vec __attribute__((ext_vector_type(N)));
  vec v;
  __device__ float operator[](int e) const { return float(v[e]); }
};
template <typename T>
struct Raw<T, 1> {
  T v;
  __device__ float operator[](int) const { return float(v); }
};

template <typename T, int N>
__device__ inline Raw<T, N> load_raw(const T *p) {
  return *reinterpret_cast<const Raw<T, N> *>(p);
}
template <typename T, int N>
__device__ inline void store_raw(T *p, const float (&x)[N]) {
  Raw<T, N> r;
  if constexpr (N == 1) r.v = T(x[0]);
  else
#pragma unroll
    for (int e = 0; e < N; ++e) r.v[e] = T(x[e]);
  *reinterpret_cast<Raw<T, N> *>(p) = r;
}

// ------------------------------------------------------------- documents -----
// What a row is: -1 of no document, else 4 times its document, + 1 if it is the
// first of it, + 2 if the last.
__device__ inline bool row_in(int info) { return info >= 0; }
__device__ inline bool row_first(int info) { return info >= 0 && (info & 1); }
__device__ inline bool row_last(int info) { return info >= 0 && (info & 2); }
// the chain is cut before it
__device__ inline bool row_cuts(int info) { return info < 0 || (info & 1); }

struct Docs {
  const int64_t *offsets;
  int64_t docs, rows;
  int cols;
  int *info;           // [rows]
  uint64_t *clear;     // words of the chain that are cleared
  int64_t clear_count;
  // empty documents: out = from (NULL = 0)
  const float *from;
  float *out;          // NULL = none
};

// The rows' documents, by a search for each row; the states of empty documents;
// and the chain's words cleared.
__global__ __launch_bounds__(256) void k_documents(const Docs d) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, step = int64_t(gridDim.x) * 256;
  for (int64_t i = at; i < d.clear_count; i += step) d.clear[i] = 0;
  for (int64_t i = at; i < d.rows; i += step) {
    int64_t low = 0, high = d.docs + 1;  // offsets that are not above i
    while (low < high) {
      const int64_t mid = (low + high) >> 1;
      if (d.offsets[mid] <= i) low = mid + 1;
      else high = mid;
    }
    const int64_t doc = low - 1;
    int info = -1;
    if (doc >= 0 && doc < d.docs) {
      const int64_t begin = d.offsets[doc], end = d.offsets[doc + 1];
      // a document that begins before the first row begins with it
      info = int(doc) * 4 + (i == begin || i == 0 ? 1 : 0) + (i + 1 == end || i + 1 == d.rows ? 2 : 0);
    }
    d.info[i] = info;
  }
  if (!d.out) return;
  for (int64_t doc = at >> 6; doc < d.docs; doc += step >> 6) {
    const int64_t begin = d.offsets[doc] > 0 ? d.offsets[doc] : 0;
    const int64_t end = d.offsets[doc + 1] < d.rows ? d.offsets[doc + 1] : d.rows;
    if (begin < end) continue;
    for (int c = threadIdx.x & 63; c < d.cols; c += 64)
      d.out[doc * d.cols + c] = d.from ? d.from[doc * d.cols + c] : 0.0f;
  }
}

// ----------------------------------------------------------------- chain -----
// What a workgroup leaves for the ones after it, for each of its columns: the
// map's A and B, and the state after its last row, each with a mark beside it in
// one word of 64 bits, so that a word is there or not.
constexpr int kWords = 3;
struct Chain {
  uint64_t *words;   // [blocks][kWords][cols]
  uint32_t *ticket;  // the workgroups' order
  int cols;
  __device__ uint64_t *at(int block, int word, int c) const {
    return words + (int64_t(block) * kWords + word) * cols + c;
  }
  __device__ void leave(int block, int word, int c, float v) const {
    __hip_atomic_store(at(block, word, c), uint64_t(1) << 32 | __builtin_bit_cast(uint32_t, v), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ uint64_t look(int block, int word, int c) const {
    return __hip_atomic_load(at(block, word, c), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

__device__ inline bool there(uint64_t word) { return word >> 32; }
__device__ inline float value(uint64_t word) { return __builtin_bit_cast(float, uint32_t(word)); }

// A workgroup's maps and what it found by looking back, of 64 N columns.
template <int N>
struct Shared {
  float a[kWaves][64 * N], b[kWaves][64 * N];
  float past_a[kWindow][64 * N], past_b[kWindow][64 * N];  // of a state: b
  int cut[kWaves];   // whether a wave's rows cut the chain
  int state[kWindow];  // whether it is a state
  int ticket;
};

// The state that comes into this wave, after the waves' maps have been left in
// `s` and synchronised: wave `order` of the workgroup's order, `block` of the
// workgroups'.  Leaves the workgroup's own map and state.  `needed`: the first
// row does not cut the chain.
//
// Waits only for workgroups of smaller tickets, which run already and leave
// their maps without waiting for anything.
template <int N>
__device__ inline void state_in(Shared<N> &s, const Chain &chain, int block, int order, bool needed, int c, bool in,
                                float (&m)[N]) {
  const int lane = threadIdx.x & 63, first = lane * N;
  // the workgroup's map, and that of the waves before this one
  float a[N], b[N], own_a[N], own_b[N];
  bool cut = false, own_cut = false;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    a[e] = own_a[e] = 1.0f;
    b[e] = own_b[e] = 0.0f;
  }
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == order) {
      own_cut = cut;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        own_a[e] = a[e];
        own_b[e] = b[e];
      }
    }
    const bool now = s.cut[w];
    cut |= now;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      b[e] = now ? s.b[w][first + e] : __builtin_fmaf(s.a[w][first + e], b[e], s.b[w][first + e]);
      a[e] *= s.a[w][first + e];
    }
  }
  const bool known = cut || block == 0;  // the state after the workgroup
  if (order == 0 && in) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (known) {
        chain.leave(block, 2, c + e, b[e]);
      } else {
        chain.leave(block, 0, c + e, a[e]);
        chain.leave(block, 1, c + e, b[e]);
      }
    }
  }
  float carry[N];
#pragma unroll
  for (int e = 0; e < N; ++e) carry[e] = 0.0f;
  if (block > 0 && needed) {  // the same in all waves
    int found;
    do {
      // each wave waits for the maps or states of kAhead workgroups before this one
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int back = order * kAhead + i, from = block - 1 - back;
        if (from < 0) {
          if (lane == 0) s.state[back] = 1;  // never reached: block 0 leaves a state
          continue;
        }
        uint64_t wa[N], wb[N], ws[N];
        bool map, state;
        do {
          map = state = true;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            wa[e] = in ? chain.look(from, 0, c + e) : 0;
            wb[e] = in ? chain.look(from, 1, c + e) : 0;
            ws[e] = in ? chain.look(from, 2, c + e) : 0;
          }
#pragma unroll
          for (int e = 0; e < N; ++e) {
            map &= !in || (there(wa[e]) && there(wb[e]));
            state &= !in || there(ws[e]);
          }
          map = !__ballot(!map);
          state = !__ballot(!state);
          if (!map && !state) __builtin_amdgcn_s_sleep(1);
        } while (!map && !state);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          s.past_a[back][first + e] = value(wa[e]);
          s.past_b[back][first + e] = state ? value(ws[e]) : value(wb[e]);
        }
        if (lane == 0) s.state[back] = state;
      }
      __syncthreads();
      found = kWindow;
#pragma unroll 4
      for (int i = kWindow - 1; i >= 0; --i) found = s.state[i] ? i : found;
      if (found == kWindow) __syncthreads();
    } while (found == kWindow);
#pragma unroll
    for (int e = 0; e < N; ++e) carry[e] = s.past_b[found][first + e];
    for (int i = found - 1; i >= 0; --i)
#pragma unroll
      for (int e = 0; e < N; ++e) carry[e] = __builtin_fmaf(s.past_a[i][first + e], carry[e], s.past_b[i][first + e]);
  }
  if (!known && order == 0 && in) {
#pragma unroll
    for (int e = 0; e < N; ++e) chain.leave(block, 2, c + e, __builtin_fmaf(a[e], carry[e], b[e]));
  }
#pragma unroll
  for (int e = 0; e < N; ++e) m[e] = own_cut ? own_b[e] : __builtin_fmaf(own_a[e], carry[e], own_b[e]);
}

// The workgroup's place in the order: workgroups of a smaller ticket run.
template <int N>
__device__ inline int take_ticket(Shared<N> &s, const Chain &chain) {
  if (threadIdx.x == 0) s.ticket = int(atomicAdd(chain.ticket, 1u));
  __syncthreads();
  return s.ticket;
}

template <typename T>
struct Forward {
  const T *x, *gate;
  int64_t ldx, ld_gate;
  const int *info;
  const float *state;
  T *h;
  int64_t ldh;
  float *last, *kept;
  int64_t rows;
  int cols, groups;
  Chain chain;
};

// Bound by its bytes: x and gate in, h out.
template <typename T, int N>
__global__ __launch_bounds__(64 * kWaves) void k_recur(const Forward<T> p) {
  __shared__ Shared<N> s;
  const int t = take_ticket(s, p.chain), block = t / p.groups;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (t % p.groups * 64 + lane) * N;
  const bool in = c < p.cols;
  const int at = in ? c : 0;
  const int64_t row0 = int64_t(block) * kBlock + wave * kRows;
  // rows past the end repeat the last one; what they are says that they are of no document
  const int mine = lane < kRows && row0 + lane < p.rows ? p.info[row0 + lane] : -1;
  Raw<T, N> x[kRows], g[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t row = row0 + r < p.rows ? row0 + r : p.rows - 1;
    x[r] = load_raw<T, N>(p.x + row * p.ldx + at);
    g[r] = load_raw<T, N>(p.gate + row * p.ld_gate + at);
  }
  float f[kRows][N], b[kRows][N];
  float a[N], sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    a[e] = 1.0f;
    sum[e] = 0.0f;
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int info = __builtin_amdgcn_readlane(mine, r);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float keep;
      gate<T>(g[r][e], f[r][e], keep);
      b[r][e] = keep * x[r][e];
    }
    if (row_cuts(info)) {
      const bool from = p.state && row_first(info);
      const float *state = p.state + int64_t(info >> 2) * p.cols + at;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (from) b[r][e] = __builtin_fmaf(f[r][e], state[e], b[r][e]);
        if (!row_in(info)) b[r][e] = 0.0f;
        sum[e] = b[r][e];
        a[e] = 0.0f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        sum[e] = __builtin_fmaf(f[r][e], sum[e], b[r][e]);
        a[e] *= f[r][e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    s.a[wave][lane * N + e] = a[e];
    s.b[wave][lane * N + e] = sum[e];
  }
  const bool cuts = __ballot(lane < kRows && row_cuts(mine));
  if (lane == 0) s.cut[wave] = cuts;
  const int begins = p.info[int64_t(block) * kBlock];
  __syncthreads();
  float m[N];
  state_in<N>(s, p.chain, block, wave, !row_cuts(begins), c, in, m);
  if (!in || row0 >= p.rows) return;
#pragma unroll
  for (int e = 0; e < N; ++e) p.kept[row0 / kRows * p.cols + c + e] = m[e];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (row0 + r >= p.rows) break;
    const int info = __builtin_amdgcn_readlane(mine, r);
    const bool cut = row_cuts(info);
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = cut ? b[r][e] : __builtin_fmaf(f[r][e], m[e], b[r][e]);
    store_raw<T, N>(p.h + (row0 + r) * p.ldh + c, m);
    if (row_last(info))
#pragma unroll
      for (int e = 0; e < N; ++e) p.last[int64_t(info >> 2) * p.cols + c + e] = m[e];
  }
}

template <typename T>
struct Backward {
  const T *x, *gate, *dh;
  int64_t ldx, ld_gate, lddh;
  const int *info;
  const float *state, *kept, *dlast;
  T *dx, *dgate;
  int64_t lddx, ld_dgate;
  float *dstate;
  int64_t rows;
  int cols, groups, blocks;
  Chain chain;
};

// The states are computed again from the kept ones, and the gradients run the
// other way: row t passes l_t g_t on to row t - 1, where l_t is f_t, or nothing
// where the chain is cut; m -> l (dh + m) is a row's map.
template <typename T, int N>
__global__ __launch_bounds__(64 * kWaves) void k_recur_backward(const Backward<T> p) {
  __shared__ Shared<N> s;
  const int t = take_ticket(s, p.chain), back = t / p.groups, block = p.blocks - 1 - back;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (t % p.groups * 64 + lane) * N;
  const bool in = c < p.cols;
  const int at = in ? c : 0;
  const int64_t row0 = int64_t(block) * kBlock + wave * kRows;
  const int mine = lane < kRows && row0 + lane < p.rows ? p.info[row0 + lane] : -1;
  Raw<T, N> x[kRows], g[kRows], d[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int64_t row = row0 + r < p.rows ? row0 + r : p.rows - 1;
    x[r] = load_raw<T, N>(p.x + row * p.ldx + at);
    g[r] = load_raw<T, N>(p.gate + row * p.ld_gate + at);
    d[r] = load_raw<T, N>(p.dh + row * p.lddh + at);
  }
  // what the state before a row is above the row's x; the rows' maps from the first row on
  float u[kRows][N], h[N], a[N], sum[N];
  const int64_t kept_row = row0 < p.rows ? row0 / kRows : 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    h[e] = p.kept[kept_row * p.cols + at + e];
    a[e] = 1.0f;
    sum[e] = 0.0f;
  }
  bool cut = false;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int info = __builtin_amdgcn_readlane(mine, r);
    if (row_cuts(info)) {
      const bool from = p.state && row_first(info);
#pragma unroll
      for (int e = 0; e < N; ++e) h[e] = from ? p.state[int64_t(info >> 2) * p.cols + at + e] : 0.0f;
      cut = true;
    }
    const bool end = p.dlast && row_last(info);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f, keep;
      gate<T>(g[r][e], f, keep);
      const float xv = x[r][e];
      u[r][e] = h[e] - xv;
      h[e] = __builtin_fmaf(f, h[e], keep * xv);
      if (!cut) {
        float dv = d[r][e];
        if (end) dv += p.dlast[int64_t(info >> 2) * p.cols + at + e];
        a[e] *= f;
        sum[e] = __builtin_fmaf(a[e], dv, sum[e]);
      }
    }
  }
  const int order = kWaves - 1 - wave;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    s.a[order][lane * N + e] = cut ? 0.0f : a[e];
    s.b[order][lane * N + e] = sum[e];
  }
  if (lane == 0) s.cut[order] = cut;
  // whether the row after the workgroup's last one passes anything on
  const int64_t after = int64_t(block + 1) * kBlock;
  const int follows = after < p.rows ? p.info[after] : -1;
  __syncthreads();
  float m[N];
  state_in<N>(s, p.chain, back, order, !row_cuts(follows), c, in, m);
  if (!in || row0 >= p.rows) return;
#pragma unroll
  for (int r = kRows - 1; r >= 0; --r) {
    if (row0 + r >= p.rows) continue;
    const int info = __builtin_amdgcn_readlane(mine, r);
    const bool inside = row_in(info), end = p.dlast && row_last(info);
    float dx[N], dg[N], next[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f, keep;
      gate<T>(g[r][e], f, keep);
      float grad = d[r][e] + m[e];
      if (end) grad += p.dlast[int64_t(info >> 2) * p.cols + c + e];
      dx[e] = inside ? keep * grad : 0.0f;
      dg[e] = inside ? grad * u[r][e] * (f * keep) : 0.0f;
      next[e] = f * grad;
    }
    store_raw<T, N>(p.dx + (row0 + r) * p.lddx + c, dx);
    store_raw<T, N>(p.dgate + (row0 + r) * p.ld_dgate + c, dg);
    const bool first = row_cuts(info);
    if (p.dstate && row_first(info))
#pragma unroll
      for (int e = 0; e < N; ++e) p.dstate[int64_t(info >> 2) * p.cols + c + e] = next[e];
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = first ? 0.0f : next[e];
  }
}

// ------------------------------------------------------------------ step -----
template <typename T, int N>
__global__ __launch_bounds__(256) void k_recur_step(const T *x, int64_t ldx, const T *gates, int64_t ldg,
                                                    const float *state, int64_t rows, int cols, T *h, int64_t ldh,
                                                    float *last) {
  const int each = (cols + N - 1) / N;
  const int64_t all = rows * each, step = int64_t(gridDim.x) * 256;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += step) {
    const int64_t row = all <= 0xffffffffll ? uint32_t(i) / uint32_t(each) : i / each;
    const int c = int(i - row * each) * N;
    const Raw<T, N> xv = load_raw<T, N>(x + row * ldx + c), gv = load_raw<T, N>(gates + row * ldg + c);
    const Raw<float, N> m = load_raw<float, N>(state + row * cols + c);
    float out[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f, keep;
      gate<T>(gv[e], f, keep);
      out[e] = __builtin_fmaf(f, m[e], keep * xv[e]);
    }
    store_raw<float, N>(last + row * cols + c, out);
    store_raw<T, N>(h + row * ldh + c, out);
  }
}

// ------------------------------------------------------------------ host -----
// Whether n columns can be moved at once.
template <typename T>
bool by(int n, const void *p, int64_t ld, int64_t cols) {
  return reinterpret_cast<uintptr_t>(p) % (n * sizeof(T)) == 0 && ld % n == 0 && cols % n == 0;
}

// The scratch of a scan over `rows`, and what finds the rows' documents.
struct Scan {
  int blocks, groups;
  int *info;
  Chain chain;
  Scan(const lda_recur_args &a, int columns, Arena &ws) {
    blocks = int(ceil_div(a.rows, kBlock));
    groups = int(ceil_div(a.cols, 64 * columns));
    info = ws.take<int>(a.rows);
    const int64_t words = int64_t(blocks) * kWords * a.cols;
    chain.words = ws.take<uint64_t>(words + 1);
    chain.ticket = reinterpret_cast<uint32_t *>(chain.words + words);
    chain.cols = a.cols;
  }
  hipError_t documents(const lda_recur_args &a, const float *from, float *out) const {
    Docs d = {};
    d.offsets = a.offsets;
    d.docs = a.docs;
    d.rows = a.rows;
    d.cols = a.cols;
    d.info = info;
    d.clear = chain.words;
    d.clear_count = int64_t(blocks) * kWords * a.cols + 1;
    d.from = from;
    d.out = out;
    int64_t most = a.rows > d.clear_count / 4 ? a.rows : d.clear_count / 4;
    if (out && a.docs * 64 > most) most = a.docs * 64;
    const int64_t needed = most > 0 ? ceil_div(most, 256) : 1;
    k_documents<<<unsigned(needed < 65536 ? needed : 65536), 256, 0, static_cast<hipStream_t>(a.stream)>>>(d);
    return hipGetLastError();
  }
};

template <typename T, int N>
hipError_t forward_n(const lda_recur_args &a, Arena &ws, bool dry) {
  const Scan scan(a, N, ws);
  if (dry) return hipSuccess;
  OPS_TRY(scan.documents(a, a.state, a.last));
  if (a.rows == 0) return hipSuccess;
  const Forward<T> p{static_cast<const T *>(a.x), static_cast<const T *>(a.gate), a.ldx, a.ld_gate, scan.info, a.state,
                     static_cast<T *>(a.h), a.ldh, a.last, a.kept, a.rows, a.cols, scan.groups, scan.chain};
  k_recur<T, N><<<unsigned(scan.blocks) * unsigned(scan.groups), 64 * kWaves, 0, static_cast<hipStream_t>(a.stream)>>>(
      p);
  return hipGetLastError();
}

template <typename T, int N>
hipError_t backward_n(const lda_recur_args &a, Arena &ws, bool dry) {
  const Scan scan(a, N, ws);
  if (dry) return hipSuccess;
  OPS_TRY(scan.documents(a, a.dlast, a.dstate));
  if (a.rows == 0) return hipSuccess;
  const Backward<T> p{static_cast<const T *>(a.x), static_cast<const T *>(a.gate), static_cast<const T *>(a.dh), a.ldx,
                      a.ld_gate, a.lddh, scan.info, a.state, a.kept, a.dlast, static_cast<T *>(a.dx),
                      static_cast<T *>(a.dgate), a.lddx, a.ld_dgate, a.dstate, a.rows, a.cols, scan.groups, scan.blocks,
                      scan.chain};
  k_recur_backward<T, N>
      <<<unsigned(scan.blocks) * unsigned(scan.groups), 64 * kWaves, 0, static_cast<hipStream_t>(a.stream)>>>(p);
  return hipGetLastError();
}

template <typename T>
hipError_t forward_t(const lda_recur_args &a, Arena &ws, bool dry) {
  if constexpr (sizeof(T) == 2) {
    if (by<T>(2, a.x, a.ldx, a.cols) && by<T>(2, a.gate, a.ld_gate, a.cols) && by<T>(2, a.h, a.ldh, a.cols))
      return forward_n<T, 2>(a, ws, dry);
  }
  return forward_n<T, 1>(a, ws, dry);
}

template <typename T>
hipError_t backward_t(const lda_recur_args &a, Arena &ws, bool dry) {
  if constexpr (sizeof(T) == 2) {
    if (by<T>(2, a.x, a.ldx, a.cols) && by<T>(2, a.gate, a.ld_gate, a.cols) && by<T>(2, a.dh, a.lddh, a.cols) &&
        by<T>(2, a.dx, a.lddx, a.cols) && by<T>(2, a.dgate, a.ld_dgate, a.cols))
      return backward_n<T, 2>(a, ws, dry);
  }
  return backward_n<T, 1>(a, ws, dry);
}

template <typename T>
hipError_t step_t(const lda_recur_args &a) {
  if (a.rows == 0) return hipSuccess;
  const auto s = static_cast<hipStream_t>(a.stream);
  const T *x = static_cast<const T *>(a.x), *g = static_cast<const T *>(a.gate);
  T *h = static_cast<T *>(a.h);
  const bool wide = by<T>(4, x, a.ldx, a.cols) && by<T>(4, g, a.ld_gate, a.cols) && by<T>(4, h, a.ldh, a.cols) &&
                    by<float>(4, a.state, a.cols, a.cols) && by<float>(4, a.last, a.cols, a.cols);
  const int64_t needed = ceil_div(a.rows * (wide ? a.cols / 4 : a.cols), 256);
  const unsigned blocks = unsigned(needed < 65536 ? needed : 65536);
  auto kernel = wide ? k_recur_step<T, 4> : k_recur_step<T, 1>;
  kernel<<<blocks, 256, 0, s>>>(x, a.ldx, g, a.ld_gate, a.state, a.rows, a.cols, h, a.ldh, a.last);
  return hipGetLastError();
}

}  // namespace

#define RECUR_BY_TYPE(fn, ...)                              \
  switch (a.dtype) {                                  \
    case LDA_F32: return fn<float>(__VA_ARGS__);      \
    case LDA_BF16: return fn<bf16>(__VA_ARGS__);      \
    default: return fn<f16>(__VA_ARGS__);             \
  }

hipError_t recur_forward(const lda_recur_args &a, Arena &ws, bool dry) { RECUR_BY_TYPE(forward_t, a, ws, dry) }
hipError_t recur_backward(const lda_recur_args &a, Arena &ws, bool dry) { RECUR_BY_TYPE(backward_t, a, ws, dry) }
hipError_t recur_step(const lda_recur_args &a) { RECUR_BY_TYPE(step_t, a) }

}  // namespace ops
}  // namespace lda
