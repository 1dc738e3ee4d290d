// Gated linear recurrence over documents (include/lda_ops.h): forward, backward
// and single steps.
//
// h_t = f_t h_{t-1} + b_t is a chain in each column.  A wave holds some rows of
// its columns in registers and reduces them to one map, state in -> state out,
// m -> A m + B; a workgroup joins its waves' maps in LDS, and workgroups, which
// start in the order of the rows, pass the state on through memory: each leaves
// its map, or, as soon as it has it, the state after its last row, looks back
// until it finds a state, and applies the maps between in their order.  So
// every input is read once and every output written once, and the results are
// those of one fixed order of the operations whichever workgroup was faster.
// A document's first row cuts the chain: a map with a first row in it does not
// depend on the state that comes in.  Scans in one pass that look back in this way
// were published by D. Merrill and M. Garland (Single-pass Parallel Prefix Scan with
// Decoupled Look-back, 2016).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace lda {
namespace ops {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kKept = LDA_OPS_RECUR_ROWS;  // rows from one kept state to the next
constexpr int kWindow = 32;                // workgroups that are looked back to at a time
constexpr int kWaves = 8;
// Rows of a wave, which has N columns a lane: as many as leave room in the
// registers for two workgroups a CU (128 a lane), so that one loads while the
// other waits or computes.  Both passes over 65536 rows x 1024 of bf16: 8 waves of
// 16 rows 278 us, 4 waves 316, 16 waves 288, 8 waves of 32 rows (one workgroup a
// CU) 318.  In single precision the backward pass' three matrices fill twice as
// many registers.
template <typename T, int N, bool Back>
constexpr int kRows = Back && sizeof(T) == 4 ? 16 : 32 / N;

constexpr float kLog2e = 1.4426950408889634f;

// The gate f = sigmoid(g) and k = 1 - f, kept as one number: the smaller of the
// two, from e = exp(-|g|) to a few roundings of itself, negative where it is f.
// The larger is 1 minus it, which no approximation of the reciprocal biases: a
// gate near 1 is multiplied by itself thousands of times.
template <typename T>
__device__ inline float gate_of(float g) {
  const float a = fabsf(g), t = -kLog2e * a;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (sizeof(T) == 4) {
    // what the product with log2 e was rounded by
    const float low = __builtin_fmaf(-kLog2e, a, -t) - 1.9259629911266175e-8f * a;
    if (a < 100.0f) e = __builtin_fmaf(e, 0.6931471805599453f * low, e);
  }
  return copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), g);
}
__device__ inline void open(float kept, float &f, float &k) {
  const float small = fabsf(kept), large = 1.0f - small;
  const bool low = __builtin_signbitf(kept);
  f = low ? small : large;
  k = low ? large : small;
}
template <typename T>
__device__ inline void gate(float g, float &f, float &k) {
  open(gate_of<T>(g), f, k);
}

// N columns of a lane, side by side, moved at once from wherever they begin.
template <typename T, int N>
struct Raw {
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
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
// Past: past the last cache, for results that it does not hold.
template <typename T, int N, bool Past = false>
__device__ inline void store_raw(T *p, const float (&x)[N]) {
  Raw<T, N> r;
  if constexpr (N == 1) r.v = T(x[0]);
  else
#pragma unroll
    for (int e = 0; e < N; ++e) r.v[e] = T(x[e]);
  if constexpr (!Past) *reinterpret_cast<Raw<T, N> *>(p) = r;
  else if constexpr (N == 1) __builtin_nontemporal_store(r.v, p);
  else __builtin_nontemporal_store(r.v, reinterpret_cast<typename Raw<T, N>::vec *>(p));
}

// Values that the compiler takes for others here: it then computes what is made
// of them where it is used, instead of keeping it in registers from earlier on.
__device__ inline void anew(float &x) { asm volatile("" : "+v"(x)); }
__device__ inline void anew(int &x) { asm volatile("" : "+v"(x)); }
template <typename T, int N>
__device__ inline void anew(Raw<T, N> &x) {
  if constexpr (sizeof(x) == 4) {
    uint32_t bits = __builtin_bit_cast(uint32_t, x);
    asm volatile("" : "+v"(bits));
    x = __builtin_bit_cast(Raw<T, N>, bits);
  }
}

// A lane's first column.  The last lane of an odd row has the last N, one of which
// its neighbour has too, and lanes past the end have them as well: all compute the
// same.
template <int N>
__device__ inline int column_of(int group, int lane, int cols) {
  return min((group * 64 + lane) * N, cols - N);
}

// A wave's lanes are P parts of 64 / P: narrow matrices leave lanes without columns
// otherwise, and a row costs a wave the same whatever its width.  Each part has R
// rows of its own, after those of the part before it.  Both passes over 262144
// rows x 20 of bf16 with 1 / 4 parts 128 / 63 us, x 64 with 1 / 2 134 / 112; one
// document x 64, forward, 190 / 101.  Addresses and what rows are then differ by
// lane and take registers, so that one workgroup fits a CU (two, with 19 registers
// in memory: x 64 124 us).
template <int P>
constexpr int kWavesPerSimd = P == 1 ? 4 : 2;
template <int P>
__device__ inline int part_of(int lane) {
  return P == 1 ? 0 : lane / (64 / P);
}
template <int P>
__device__ inline int lane_of(int lane) {
  return P == 1 ? lane : lane & (64 / P - 1);
}
// Whether a lane goes on to what is stored.  A whole wave reads what its rows are from
// the registers of other lanes (doc_of), so all of its lanes have to be there to the
// end: those past the end of a row leave, look for and store what the last one does.
template <int N, int P>
__device__ inline bool lane_in(int group, int lane, int cols) {
  return P == 1 || (group * 64 + lane_of<P>(lane)) * N < cols;
}

// ------------------------------------------------------------- documents -----
// What a row is: -1 of no document, else 4 times its document, + 1 if it is the
// first of it, + 2 if the last.
__device__ inline bool row_cuts(int info) { return info < 0 || (info & 1); }

// The rows of a part of a wave that are not inside a document: one bit a row.
// Lane p R + r has what row r of part p is, other lanes -1.
struct Special {
  uint32_t outs, cuts, lasts;
  __device__ Special(int info, int rows, int part)
      : outs(uint32_t(__ballot(info < 0) >> part * rows)), cuts(uint32_t(__ballot(row_cuts(info)) >> part * rows)),
        lasts(uint32_t(__ballot(info >= 0 && (info & 2)) >> part * rows)) {
    const uint32_t all = uint32_t((uint64_t(1) << rows) - 1);
    outs &= all;
    cuts &= all;
    lasts &= all;
  }
  __device__ bool out(int r) const { return outs >> r & 1; }    // of no document
  __device__ bool cut(int r) const { return cuts >> r & 1; }    // the chain is cut before it
  __device__ bool first(int r) const { return (cuts & ~outs) >> r & 1; }
  __device__ bool last(int r) const { return lasts >> r & 1; }
};

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

// How many offsets are not above `row`, the same in all lanes: the wave looks at
// 64 places at a time.
__device__ inline int64_t offsets_upto(const Docs &d, int64_t row, int lane) {
  int64_t low = 0, high = d.docs + 1;
  while (low < high) {
    const int64_t step = (high - low + 63) >> 6, at = low + (lane + 1) * step - 1;
    const uint64_t upto = __ballot(at < high && d.offsets[at] <= row);
    // in order: the first ones
    const int64_t next = low + __popcll(upto) * step;
    if (step == 1) return next;
    high = next + step - 1 < high ? next + step - 1 : high;
    low = next;
  }
  return low;
}

// The rows' documents, 64 rows a wave: a search for the first one, and the next
// offsets from there; rows of more than 64 documents (many of them empty) are
// searched for one by one.  And the states of empty documents, and the chain's
// words cleared.
__global__ __launch_bounds__(256) void k_documents(const Docs d) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, step = int64_t(gridDim.x) * 256;
  const int lane = threadIdx.x & 63;
  for (int64_t i = at; i < d.clear_count; i += step) d.clear[i] = 0;
  for (int64_t row0 = at - lane; row0 < d.rows; row0 += step) {
    const int64_t upto = offsets_upto(d, row0, lane), row = row0 + lane;
    const int64_t next = upto + lane <= d.docs ? d.offsets[upto + lane] - row0 : 65;
    const int rel = next > 65 ? 65 : next < 0 ? 0 : int(next);  // of the offsets after the first row's
    int64_t doc, begin, end;
    if (__shfl(rel, 63) > 63) {
      int count = 0;  // of them, not above the row
#pragma unroll
      for (int x = 32; x > 0; x >>= 1)
        if (__shfl(rel, count + x - 1) <= lane) count += x;
      doc = upto - 1 + count;
      const int before = __shfl(rel, count - 1 < 0 ? 0 : count - 1), after = __shfl(rel, count);
      begin = count > 0 ? row0 + before : upto > 0 ? d.offsets[upto - 1] : 0;
      end = row0 + after;
    } else {
      int64_t low = upto, high = d.docs + 1;
      while (low < high) {
        const int64_t mid = (low + high) >> 1;
        if (d.offsets[mid] <= row) low = mid + 1;
        else high = mid;
      }
      doc = low - 1;
      begin = doc >= 0 ? d.offsets[doc] : 0;
      end = doc >= 0 && doc < d.docs ? d.offsets[doc + 1] : 0;
    }
    if (row >= d.rows) continue;
    int info = -1;
    // a document that begins before the first row begins with it
    if (doc >= 0 && doc < d.docs)
      info = int(doc) * 4 + (row == begin || row == 0 ? 1 : 0) + (row + 1 == end || row + 1 == d.rows ? 2 : 0);
    d.info[row] = info;
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
// What a workgroup leaves for the ones after it, in two words of 64 bits for each
// of its lanes' columns: its map's A and B, and in the place of B, as soon as it
// has it, the state after its last row.  A word holds its value and beside it what
// it is, so that a reader needs no order between the words.  They are numbered by
// the lanes, not by the columns: a column that two workgroups have (column_of) has
// words of each, or the map of one could take the place of the other's state.
enum : uint32_t { kNothing = 0, kMap = 1, kState = 2 };
constexpr int kWords = 2;
struct Chain {
  uint64_t *words;   // [blocks][kWords][slots]
  uint32_t *ticket;  // the workgroups' order
  int slots;         // N for each lane of the workgroups of a row
  // the workgroup's slots begin at `part`, `slot` is a lane's among them
  __device__ uint64_t *at(int block, int word, int part, int slot) const {
    return words + ((int64_t(block) * kWords + word) * slots + part) + slot;
  }
  __device__ void leave(int block, int word, int part, int slot, uint32_t what, float v) const {
    __hip_atomic_store(at(block, word, part, slot), uint64_t(what) << 32 | __builtin_bit_cast(uint32_t, v), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
  }
  __device__ uint64_t look(int block, int word, int part, int slot) const {
    return __hip_atomic_load(at(block, word, part, slot), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
};

__device__ inline uint32_t what(uint64_t word) { return uint32_t(word >> 32); }
__device__ inline float value(uint64_t word) { return __builtin_bit_cast(float, uint32_t(word)); }

// A workgroup's maps and what it found by looking back, of 64 N columns.
template <int N>
struct Shared {
  float a[kWaves][64 * N], b[kWaves][64 * N];
  float past_a[kWindow][64 * N], past_b[kWindow][64 * N];  // of a state: b
  int cut[kWaves];  // whether a wave's rows cut the chain
  int nearest;      // the state among the past that is nearest, kWindow if there is none
  int ticket;
};

// What a wave has seen of another workgroup's words.
template <int N>
struct Look {
  uint64_t a[N], b[N];
  __device__ void take(const Chain &chain, int from, int word, int part, int slot, bool in) {
#pragma unroll
    for (int e = 0; e < N; ++e) (word ? b : a)[e] = in ? chain.look(from, word, part, slot + e) : 0;
  }
  __device__ bool all(const uint64_t (&w)[N], uint32_t is, bool in) const {
    bool yes = true;
#pragma unroll
    for (int e = 0; e < N; ++e) yes &= !in || what(w[e]) == is;
    return !__ballot(!yes);
  }
};

// The state that comes into this wave, whose rows' map is (a, b) and cuts the
// chain or not: wave `order` of the workgroup's order, `block` of the
// workgroups'.  Leaves the workgroup's own map and state.  `needed`: the
// workgroup's first row does not cut the chain.
//
// Waits only for workgroups of smaller tickets, which run already: they leave
// their maps without waiting for anything, and their states once the one before
// them has (the first at once).  A look at memory takes 1.5 us in a
// full machine, as long as a sixth of a workgroup's life, and 2 KiB of all
// columns' words: a wave looks at one word until it knows that it needs the others
// (when both passes over 65536 rows x 1024 of bf16 took 306 us, all columns at each
// look took 366, and a first look before the workgroup's maps are joined 362).
template <int N, int P>
__device__ inline void state_in(Shared<N> &s, const Chain &chain, int block, int order, bool needed, int group, bool in,
                                const float (&map_a)[N], const float (&map_b)[N], bool cuts, float (&m)[N]) {
  const int lane = threadIdx.x & 63, first = lane_of<P>(lane) * N, part = group * 64 * N;
  const bool leaves = in && part_of<P>(lane) == 0;
  needed &= block > 0;  // the same in all waves
#pragma unroll
  for (int e = 0; e < N; ++e) {
    s.a[order][first + e] = map_a[e];
    s.b[order][first + e] = map_b[e];
  }
  if (lane == 0) s.cut[order] = cuts;
  __syncthreads();
  // the map of the waves before this one; the first wave's turn is the whole workgroup's
  float a[N], b[N];
  bool cut = false;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    a[e] = 1.0f;
    b[e] = 0.0f;
  }
  const uint32_t all_cuts = uint32_t(__ballot(lane < kWaves && s.cut[lane & (kWaves - 1)]));
  const int waves = order == 0 ? kWaves : order;
  for (int w0 = 0; w0 < waves; w0 += 4) {
    float wa[4][N], wb[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        wa[i][e] = s.a[w0 + i][first + e];
        wb[i][e] = s.b[w0 + i][first + e];
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in_turn = w0 + i < waves, now = in_turn && (all_cuts >> (w0 + i) & 1);
      cut |= now;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float next = __builtin_fmaf(wa[i][e], now ? 0.0f : b[e], wb[i][e]);
        b[e] = in_turn ? next : b[e];
        a[e] = in_turn ? a[e] * wa[i][e] : a[e];
      }
    }
  }
  const bool known = cut || block == 0;  // the state after the workgroup, in its first wave
  if (order == 0 && leaves) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (!known) chain.leave(block, 0, part, first + e, kMap, a[e]);
      chain.leave(block, 1, part, first + e, known ? kState : kMap, b[e]);
    }
  }
  float carry[N];
#pragma unroll
  for (int e = 0; e < N; ++e) carry[e] = 0.0f;
  if (needed) {
    int found;
    while (true) {
      // each wave looks at every kWaves-th workgroup before this one, until it or another wave has a state that is
      // nearer than what it waits for
      for (int back = order; back < kWindow && back < block; back += kWaves) {
        const int from = block - 1 - back;
        Look<N> seen;
        bool state = false;
        while (true) {
          const uint32_t peek = __builtin_amdgcn_readfirstlane(what(chain.look(from, 1, part, 0)));
          if (peek == kState && lane == 0) atomicMin(&s.nearest, back);
          if (__hip_atomic_load(&s.nearest, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < back) break;
          if (peek == kNothing) {
            __builtin_amdgcn_s_sleep(2);
            continue;
          }
          seen.take(chain, from, 1, part, first, in);
          state = seen.all(seen.b, kState, in);
          if (state) break;
          if (seen.all(seen.b, kMap, in)) {
            seen.take(chain, from, 0, part, first, in);
            if (seen.all(seen.a, kMap, in)) break;
          }
        }
        if (!state && __hip_atomic_load(&s.nearest, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) < back) break;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          s.past_a[back][first + e] = value(seen.a[e]);
          s.past_b[back][first + e] = value(seen.b[e]);
        }
        if (state) {
          // the word that was peeked at may have been a map then
          if (lane == 0) atomicMin(&s.nearest, back);
          break;
        }
      }
      __syncthreads();
      found = s.nearest;
      if (found < kWindow) break;
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < N; ++e) carry[e] = s.past_b[found][first + e];
    for (int i = found - 1; i >= 0; --i)
#pragma unroll
      for (int e = 0; e < N; ++e) carry[e] = __builtin_fmaf(s.past_a[i][first + e], carry[e], s.past_b[i][first + e]);
  }
  if (order == 0) {
    if (!known && leaves) {
#pragma unroll
      for (int e = 0; e < N; ++e) chain.leave(block, 1, part, first + e, kState, __builtin_fmaf(a[e], carry[e], b[e]));
    }
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = carry[e];
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = cut ? b[e] : __builtin_fmaf(a[e], carry[e], b[e]);
  }
}

// The maps of a wave's parts, (a, b) and whether one cuts the chain, joined from the
// first part on (Back: from the last): (a, b) becomes the whole wave's, and before is
// what comes to this part of the state that comes to the wave.
template <int N, int P, bool Back>
struct Parts {
  float a[N], b[N];
  bool cut;
  __device__ Parts(float (&map_a)[N], float (&map_b)[N], bool &cuts) {
    if constexpr (P == 1) return;
    constexpr int L = 64 / P;
    const int lane = threadIdx.x & 63, turn = Back ? P - 1 - part_of<P>(lane) : part_of<P>(lane);
    auto from = [&](auto v, int by) { return Back ? __shfl_down(v, by) : __shfl_up(v, by); };
#pragma unroll
    for (int x = 1; x < P; x <<= 1) {
      const bool joins = turn >= x, other = from(int(cuts), x * L);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float pa = from(map_a[e], x * L), pb = from(map_b[e], x * L);
        if (joins && !cuts) {
          map_b[e] = __builtin_fmaf(map_a[e], pb, map_b[e]);
          map_a[e] *= pa;
        }
      }
      cuts |= joins && other;
    }
    cut = from(int(cuts), L) && turn > 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      a[e] = from(map_a[e], L);
      b[e] = from(map_b[e], L);
      if (turn == 0) {
        a[e] = 1.0f;
        b[e] = 0.0f;
      }
    }
    const int whole = (Back ? 0 : P - 1) * L + lane_of<P>(lane);
    cuts = __shfl(int(cuts), whole);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      map_a[e] = __shfl(map_a[e], whole);
      map_b[e] = __shfl(map_b[e], whole);
    }
  }
  __device__ void apply(float (&m)[N]) const {
    if constexpr (P > 1)
#pragma unroll
      for (int e = 0; e < N; ++e) m[e] = cut ? b[e] : __builtin_fmaf(a[e], m[e], b[e]);
  }
};

// The document of row r of a part.
template <int P>
__device__ inline int64_t doc_of(int mine, const int *info, int row0, int r) {
  return (P == 1 ? __builtin_amdgcn_readlane(mine, r) : info[row0 + r]) >> 2;
}

// The workgroup's place in the order: workgroups of a smaller ticket run.
template <int N>
__device__ inline int take_ticket(Shared<N> &s, const Chain &chain) {
  if (threadIdx.x == 0) {
    s.ticket = int(atomicAdd(chain.ticket, 1u));
    s.nearest = kWindow;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(s.ticket);
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
  int rows, cols, groups;
  Chain chain;
};

// Bound by its bytes, x and gate in and h out, with an eighth of h more in the kept
// states and a tenth of the time in looking back: 65536 rows x 1024 of bf16 99 us
// = 4.1 TB/s of x, gate and h (a copy reaches 4.8), 262144 x 1000 of f16 389 us =
// 4.0; one document of 65537 rows x 257 in single precision, where every workgroup
// waits for the state of those before it, 67 us = 3.0.
template <typename T, int N, int P, bool Past>
__global__ __launch_bounds__(64 * kWaves, kWavesPerSimd<P>) void k_recur(const Forward<T> p) {
  constexpr int R = kRows<T, N, false>;
  __shared__ Shared<N> s;
  const int t = take_ticket(s, p.chain), block = t / p.groups;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool in = lane_in<N, P>(t % p.groups, lane, p.cols);
  const int c = column_of<N>(t % p.groups, lane_of<P>(lane), p.cols);
  const int wave_row = (block * kWaves + wave) * R * P, row0 = wave_row + part_of<P>(lane) * R;
  // rows past the end repeat the last one; what they are says that they are of no document
  const int mine = lane < R * P && wave_row + lane < p.rows ? p.info[wave_row + lane] : -1;
  const int begins = p.info[block * R * P * kWaves];
  Raw<T, N> x[R], g[R];
  const int last_row = p.rows - 1;
  const T *px = p.x + int64_t(min(row0, last_row)) * p.ldx, *pg = p.gate + int64_t(min(row0, last_row)) * p.ld_gate;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    x[r] = load_raw<T, N>(px + c);
    g[r] = load_raw<T, N>(pg + c);
    px += row0 + r < last_row ? p.ldx : 0;
    pg += row0 + r < last_row ? p.ld_gate : 0;
  }
  float f[R][N], b[R][N];
  float a[N], sum[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    a[e] = 1.0f;
    sum[e] = 0.0f;
  }
  const Special special(mine, R, part_of<P>(lane));
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool cut = special.cut(r);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float keep;
      gate<T>(g[r][e], f[r][e], keep);
      b[r][e] = keep * x[r][e];
    }
    if (special.first(r) && p.state) {
      const float *state = p.state + doc_of<P>(mine, p.info, row0, r) * p.cols + c;
#pragma unroll
      for (int e = 0; e < N; ++e) b[r][e] = __builtin_fmaf(f[r][e], state[e], b[r][e]);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (special.out(r)) b[r][e] = 0.0f;
      f[r][e] = cut ? 0.0f : f[r][e];
      sum[e] = __builtin_fmaf(f[r][e], cut ? 0.0f : sum[e], b[r][e]);
      a[e] = cut ? 0.0f : a[e] * f[r][e];  // a document before may have a gate that is NaN
    }
  }
  float m[N];
  bool cuts = special.cuts != 0;
  const Parts<N, P, false> before(a, sum, cuts);
  state_in<N, P>(s, p.chain, block, wave, !row_cuts(begins), t % p.groups, in, a, sum, cuts, m);
  before.apply(m);
  if (!in || row0 >= p.rows) return;
  T *h = p.h + int64_t(row0) * p.ldh;
  float *kept = p.kept + int64_t(row0 / kKept) * p.cols;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (row0 + r >= p.rows) continue;
    if (r % kKept == 0) store_raw<float, N>(kept + int64_t(r / kKept) * p.cols + c, m);
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = __builtin_fmaf(f[r][e], special.cut(r) ? 0.0f : m[e], b[r][e]);
    store_raw<T, N, Past>(h + c, m);
    h += p.ldh;
    if (special.last(r)) {
      float *last = p.last + doc_of<P>(mine, p.info, row0, r) * p.cols + c;
#pragma unroll
      for (int e = 0; e < N; ++e) last[e] = m[e];
    }
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
  int rows, cols, groups, blocks;
  Chain chain;
};

// The states are computed again from the kept ones, and the gradients run the
// other way: row t passes l_t g_t on to row t - 1, where l_t is f_t, or nothing
// where the chain is cut; m -> l (dh + m) is a row's map.  65536 rows x 1024 of
// bf16: 165 us = 4.1 TB/s of x, gate, dh, dx and dgate; 65537 x 257 in single
// precision 104 us = 3.2.
template <typename T, int N, int P, bool Past>
__global__ __launch_bounds__(64 * kWaves, kWavesPerSimd<P>) void k_recur_backward(const Backward<T> p) {
  constexpr int R = kRows<T, N, true>;
  __shared__ Shared<N> s;
  const int t = take_ticket(s, p.chain), back = t / p.groups, block = p.blocks - 1 - back;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool in = lane_in<N, P>(t % p.groups, lane, p.cols);
  int c = column_of<N>(t % p.groups, lane_of<P>(lane), p.cols);
  const int wave_row = (block * kWaves + wave) * R * P, row0 = wave_row + part_of<P>(lane) * R;
  const int mine = lane < R * P && wave_row + lane < p.rows ? p.info[wave_row + lane] : -1;
  // whether the row after the workgroup's last one passes anything on
  const int after = (block + 1) * R * P * kWaves;
  const int follows = after < p.rows ? p.info[after] : -1;
  Raw<T, N> x[R], g[R], d[R];
  const int last_row = p.rows - 1;
  const T *px = p.x + int64_t(min(row0, last_row)) * p.ldx, *pg = p.gate + int64_t(min(row0, last_row)) * p.ld_gate;
  const T *pd = p.dh + int64_t(min(row0, last_row)) * p.lddh;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    x[r] = load_raw<T, N>(px + c);
    g[r] = load_raw<T, N>(pg + c);
    d[r] = load_raw<T, N>(pd + c);
    px += row0 + r < last_row ? p.ldx : 0;
    pg += row0 + r < last_row ? p.ld_gate : 0;
    pd += row0 + r < last_row ? p.lddh : 0;
  }
  // the rows' gates, and what a row's gradient is multiplied by for dgate; their maps from the first row on
  float z[R][N], w[R][N], h[N], a[N], sum[N];
  const int64_t kept_row = row0 < p.rows ? row0 / kKept : 0;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    h[e] = p.kept[kept_row * p.cols + c + e];
    a[e] = 1.0f;
    sum[e] = 0.0f;
  }
  const Special special(mine, R, part_of<P>(lane));
  // only the first of the part's last rows may lie before a cut
  const int last = p.dlast && special.lasts ? __ffs(int(special.lasts)) - 1 : -1;
  float more[N];
#pragma unroll
  for (int e = 0; e < N; ++e)
    more[e] = last < 0 ? 0.0f : p.dlast[doc_of<P>(mine, p.info, row0, last) * p.cols + c + e];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (special.cut(r)) {
#pragma unroll
      for (int e = 0; e < N; ++e) h[e] = 0.0f;
      if (special.first(r) && p.state)
#pragma unroll
        for (int e = 0; e < N; ++e)
          h[e] = p.state[doc_of<P>(mine, p.info, row0, r) * p.cols + c + e];
    }
    const bool cut = special.cuts << (31 - r);  // this row or one before it: its part goes to no row before them
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f, k;
      z[r][e] = gate_of<T>(g[r][e]);
      open(z[r][e], f, k);
      const float xv = x[r][e];
      w[r][e] = (h[e] - xv) * (f * k);
      anew(w[r][e]);
      h[e] = __builtin_fmaf(f, h[e], k * xv);
      a[e] = cut ? 0.0f : a[e] * f;
      sum[e] = cut ? sum[e] : __builtin_fmaf(a[e], r == last ? d[r][e] + more[e] : d[r][e], sum[e]);
    }
  }
  const int order = kWaves - 1 - wave;
  float m[N];
  bool cuts = special.cuts != 0;
  const Parts<N, P, true> before(a, sum, cuts);
  state_in<N, P>(s, p.chain, back, order, !row_cuts(follows), t % p.groups, in, a, sum, cuts, m);
  before.apply(m);
  if (!in || row0 >= p.rows) return;
  // the column once more: kept in a register until here it would send others to memory
  int again = threadIdx.x & 63;
  anew(again);
  c = column_of<N>(t % p.groups, lane_of<P>(again), p.cols);
  T *dx_row = p.dx + int64_t(row0 + R) * p.lddx, *dg_row = p.dgate + int64_t(row0 + R) * p.ld_dgate;
#pragma unroll
  for (int r = R - 1; r >= 0; --r) {
    dx_row -= p.lddx;
    dg_row -= p.ld_dgate;
    if (row0 + r >= p.rows) continue;
    float dx[N], dg[N];
    anew(d[r]);
    // nothing comes to a last row from the next one
    if (special.last(r) && p.dlast)
#pragma unroll
      for (int e = 0; e < N; ++e) m[e] = p.dlast[doc_of<P>(mine, p.info, row0, r) * p.cols + c + e];
    const bool out = special.out(r);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float f, k;
      anew(z[r][e]);
      open(z[r][e], f, k);
      const float grad = d[r][e] + m[e];
      dx[e] = out ? 0.0f : k * grad;
      dg[e] = out ? 0.0f : w[r][e] * grad;
      m[e] = f * grad;
    }
    store_raw<T, N, Past>(dx_row + c, dx);
    store_raw<T, N, Past>(dg_row + c, dg);
    if (special.first(r) && p.dstate)
#pragma unroll
      for (int e = 0; e < N; ++e) p.dstate[doc_of<P>(mine, p.info, row0, r) * p.cols + c + e] = m[e];
#pragma unroll
    for (int e = 0; e < N; ++e) m[e] = special.cut(r) ? 0.0f : m[e];
  }
}

// ------------------------------------------------------------------ step -----
// N columns a lane, of which a row is a multiple: the new state may take the place
// of the old one, so no column is computed twice.
template <typename T, int N>
__global__ __launch_bounds__(256) void k_recur_step(const T *x, int64_t ldx, const T *gates, int64_t ldg,
                                                    const float *state, int64_t rows, int cols, T *h, int64_t ldh,
                                                    float *last) {
  const int each = cols / N;
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
// The scratch of a scan over `rows`, and what finds the rows' documents.
struct Scan {
  int blocks, groups;
  int *info;
  Chain chain;
  Scan(const lda_recur_args &a, int columns, int rows_each, Arena &ws) {
    blocks = int(ceil_div(a.rows, rows_each));
    groups = int(ceil_div(a.cols, 64 * columns));
    info = ws.take<int>(a.rows);
    chain.slots = groups * 64 * columns;
    const int64_t words = int64_t(blocks) * kWords * chain.slots;
    chain.words = ws.take<uint64_t>(words + 1);
    chain.ticket = reinterpret_cast<uint32_t *>(chain.words + words);
  }
  hipError_t documents(const lda_recur_args &a, const float *from, float *out) const {
    Docs d = {};
    d.offsets = a.offsets;
    d.docs = a.docs;
    d.rows = a.rows;
    d.cols = a.cols;
    d.info = info;
    d.clear = chain.words;
    d.clear_count = int64_t(blocks) * kWords * chain.slots + 1;
    d.from = from;
    d.out = out;
    int64_t most = a.rows > d.clear_count / 4 ? a.rows : d.clear_count / 4;
    if (out && a.docs * 64 > most) most = a.docs * 64;
    const int64_t needed = most > 0 ? ceil_div(most, 256) : 1;
    k_documents<<<unsigned(needed < 65536 ? needed : 65536), 256, 0, static_cast<hipStream_t>(a.stream)>>>(d);
    return hipGetLastError();
  }
};

// Whether the results, of so many bytes a row and column, are stored past the last
// cache of 256 MB: 262144 x 1000 of f16 404 -> 395 us, both passes over 65536 x 1024
// of bf16 275 -> 269.  Smaller ones are left there for who reads them next.
bool past_cache(const lda_recur_args &a, size_t bytes) {
  return a.rows * a.cols * int64_t(bytes) >= int64_t(256) << 20;
}

template <typename T, int N, int P>
hipError_t forward_n(const lda_recur_args &a, Arena &ws, bool dry) {
  const Scan scan(a, N, kRows<T, N, false> * P * kWaves, ws);
  if (dry) return hipSuccess;
  OPS_TRY(scan.documents(a, a.state, a.last));
  if (a.rows == 0) return hipSuccess;
  const Forward<T> p{static_cast<const T *>(a.x), static_cast<const T *>(a.gate), a.ldx, a.ld_gate, scan.info, a.state,
                     static_cast<T *>(a.h), a.ldh, a.last, a.kept, int(a.rows), a.cols, scan.groups, scan.chain};
  auto kernel = P == 1 && past_cache(a, sizeof(T)) ? k_recur<T, N, P, P == 1> : k_recur<T, N, P, false>;
  kernel<<<unsigned(scan.blocks) * unsigned(scan.groups), 64 * kWaves, 0, static_cast<hipStream_t>(a.stream)>>>(
      p);
  return hipGetLastError();
}

template <typename T, int N, int P>
hipError_t backward_n(const lda_recur_args &a, Arena &ws, bool dry) {
  const Scan scan(a, N, kRows<T, N, true> * P * kWaves, ws);
  if (dry) return hipSuccess;
  OPS_TRY(scan.documents(a, a.dlast, a.dstate));
  if (a.rows == 0) return hipSuccess;
  const Backward<T> p{static_cast<const T *>(a.x), static_cast<const T *>(a.gate), static_cast<const T *>(a.dh), a.ldx,
                      a.ld_gate, a.lddh, scan.info, a.state, a.kept, a.dlast, static_cast<T *>(a.dx),
                      static_cast<T *>(a.dgate), a.lddx, a.ld_dgate, a.dstate, int(a.rows), a.cols, scan.groups, scan.blocks,
                      scan.chain};
  auto kernel = P == 1 && past_cache(a, 2 * sizeof(T)) ? k_recur_backward<T, N, P, P == 1>
                                                        : k_recur_backward<T, N, P, false>;
  kernel<<<unsigned(scan.blocks) * unsigned(scan.groups), 64 * kWaves, 0, static_cast<hipStream_t>(a.stream)>>>(p);
  return hipGetLastError();
}

// Calls fn with the columns of a lane (16-bit ones in pairs, 32 bits as in single
// precision) and the parts of a wave: as many as a row leaves room for and as the
// wave has lanes to hold what their rows are.
template <typename T, bool Back, typename Fn>
hipError_t with_lanes(int cols, Fn fn) {
  auto parts = [&](auto n) {
    constexpr int N = decltype(n)::value, R = kRows<T, N, Back>;
    if constexpr (R * 4 <= 64) {
      if (cols <= 16 * N) return fn(n, std::integral_constant<int, 4>());
    }
    if constexpr (R * 2 <= 64) {
      if (cols <= 32 * N) return fn(n, std::integral_constant<int, 2>());
    }
    return fn(n, std::integral_constant<int, 1>());
  };
  if constexpr (sizeof(T) == 2) {
    if (cols > 1) return parts(std::integral_constant<int, 2>());
  }
  return parts(std::integral_constant<int, 1>());
}

template <typename T>
hipError_t forward_t(const lda_recur_args &a, Arena &ws, bool dry) {
  return with_lanes<T, false>(a.cols, [&](auto n, auto p) {
    return forward_n<T, decltype(n)::value, decltype(p)::value>(a, ws, dry);
  });
}

template <typename T>
hipError_t backward_t(const lda_recur_args &a, Arena &ws, bool dry) {
  return with_lanes<T, true>(a.cols, [&](auto n, auto p) {
    return backward_n<T, decltype(n)::value, decltype(p)::value>(a, ws, dry);
  });
}

template <typename T>
hipError_t step_t(const lda_recur_args &a) {
  if (a.rows == 0) return hipSuccess;
  const auto s = static_cast<hipStream_t>(a.stream);
  const T *x = static_cast<const T *>(a.x), *g = static_cast<const T *>(a.gate);
  T *h = static_cast<T *>(a.h);
  const bool wide = a.cols % 4 == 0;
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
