// Word embedding and its gradient (include/lda_ops.h).
//
// The forward pass copies rows of the table.  The backward pass sorts the rows
// of dy by word, so that a word's gradient is a sum over neighbours in the
// order, and sums pieces of a fixed number of sorted rows: a word that is a
// tenth of the corpus then costs no more than its rows, and no sum depends on
// the order in which workgroups run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace lda {
namespace ops {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

template <typename T, int N>
using Vec = T __attribute__((ext_vector_type(N)));

// N neighbours of a row from column c on, which are moved at once (N > 1: the
// rows start at multiples of their bytes and hold a multiple of N).
template <typename T, int N>
struct Some {
  T v[N];
  __device__ void load(const T *p) {
    if constexpr (N == 1) {
      v[0] = *p;
    } else {
      const Vec<T, N> w = *reinterpret_cast<const Vec<T, N> *>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = w[e];
    }
  }
  __device__ void store(T *p) const {
    if constexpr (N == 1) {
      *p = v[0];
    } else {
      Vec<T, N> w;
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = v[e];
      *reinterpret_cast<Vec<T, N> *>(p) = w;
    }
  }
};

// -------------------------------------------------------------- forward -----
// 2^shift lanes a row (a workgroup has 256 >> shift rows at a time), four rows
// of each lane in flight.
template <typename T, int N>
__global__ __launch_bounds__(256) void k_embed(const int32_t *words, int64_t rows, const T *weight, int64_t ldw,
                                               int width, int vocab, float scale, int shift, T *y, int64_t ldy) {
  constexpr int U = 4;
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), each = 256 >> shift;
  const int64_t first = int64_t(blockIdx.x) * each * U + (threadIdx.x >> shift);
  int word[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = first + u * each;
    word[u] = i < rows ? words[i] : -1;
  }
  for (int c = lane * N; c < width; c += lanes * N) {
    Some<T, N> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[u].v[e] = T(0.0f);
      if (word[u] >= 0 && word[u] < vocab) v[u].load(weight + int64_t(word[u]) * ldw + c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = first + u * each;
      if (i >= rows) break;
      // a row of no word is 0 whatever the scale
#pragma unroll
      for (int e = 0; e < N; ++e) v[u].v[e] = T(float(v[u].v[e]) * scale);
      v[u].store(y + i * ldy + c);
    }
  }
}

// ------------------------------------------------------------------ sort -----
// Keys are the words, and `vocab` for places of no word, which so come last.
__device__ inline uint32_t key_of(int32_t word, uint32_t vocab) {
  return uint32_t(word) < vocab ? uint32_t(word) : vocab;
}

// Up to kSmall places in one workgroup: a bitonic network over (key, place),
// which no two places share, so the order is the stable one.
constexpr int kSmall = 8192;
__global__ __launch_bounds__(1024) void k_sort_small(const int32_t *words, int n, int padded, uint32_t vocab,
                                                     uint32_t *keys, uint32_t *places) {
  __shared__ uint64_t all[kSmall];
  for (int i = threadIdx.x; i < padded; i += 1024)
    all[i] = i < n ? uint64_t(key_of(words[i], vocab)) << 32 | uint32_t(i) : ~uint64_t(0);
  for (int size = 2; size <= padded; size <<= 1)
    for (int apart = size >> 1; apart > 0; apart >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < padded / 2; i += 1024) {
        const int low = (i & ~(apart - 1)) * 2 + (i & (apart - 1)), high = low + apart;
        const uint64_t a = all[low], b = all[high];
        if ((a > b) == ((low & size) == 0)) {
          all[low] = b;
          all[high] = a;
        }
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 1024) {
    keys[i] = uint32_t(all[i] >> 32);
    places[i] = uint32_t(all[i]);
  }
}

// More: a radix sort from the lowest digit of up to kDigitBits bits on, three
// launches a digit: counts of each tile, their sums before each tile, and the
// tile's places moved to where they belong, in their order.
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits, kTile = 2048;

struct SortPass {
  const int32_t *words;  // of the first pass: keys from the words, places 0, 1, ..
  const uint32_t *keys, *places;
  uint32_t *keys_out, *places_out;
  int64_t n;
  uint32_t vocab;
  int shift, bits;
  int64_t tiles;
  uint32_t *counts;  // [digits][tiles], then the digits' totals
  __device__ uint32_t key(int64_t i) const { return words ? key_of(words[i], vocab) : keys[i]; }
  __device__ uint32_t digit(uint32_t key) const { return key >> shift & ((1u << bits) - 1); }
};

__global__ __launch_bounds__(256) void k_sort_count(const SortPass p) {
  __shared__ uint32_t count[kDigits];
  const int digits = 1 << p.bits;
  for (int d = threadIdx.x; d < digits; d += 256) count[d] = 0;
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * kTile;
  for (int i = threadIdx.x; i < kTile; i += 256)
    if (first + i < p.n) atomicAdd(&count[p.digit(p.key(first + i))], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += 256) p.counts[d * p.tiles + blockIdx.x] = count[d];
}

// The sum of the values of the threads before this one; `total` of all 256.
__device__ inline uint32_t sum_before(uint32_t v, uint32_t &total, uint32_t (&shared)[4]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    const uint32_t other = __shfl_up(upto, x);
    if (lane >= x) upto += other;
  }
  __syncthreads();
  if (lane == 63) shared[wave] = upto;
  __syncthreads();
  uint32_t before = upto - v;
  total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) before += shared[w];
    total += shared[w];
  }
  return before;
}

// A digit's counts become the sums of the tiles before; one workgroup a digit.
__global__ __launch_bounds__(256) void k_sort_sums(const SortPass p) {
  __shared__ uint32_t shared[4];
  uint32_t *row = p.counts + int64_t(blockIdx.x) * p.tiles, carry = 0;
  for (int64_t t0 = 0; t0 < p.tiles; t0 += 256) {
    const int64_t t = t0 + threadIdx.x;
    const uint32_t v = t < p.tiles ? row[t] : 0;
    uint32_t total;
    const uint32_t before = sum_before(v, total, shared);
    if (t < p.tiles) row[t] = carry + before;
    carry += total;
  }
  if (threadIdx.x == 0) p.counts[(int64_t(1) << p.bits) * p.tiles + blockIdx.x] = carry;
}

// Each wave takes a quarter of the tile, 64 places at a time: a place's rank
// among those of its digit is the number of lanes before it with the same one,
// found by one ballot a bit, and what its wave had of them already.
__global__ __launch_bounds__(256) void k_sort_place(const SortPass p) {
  constexpr int ROUNDS = kTile / 256;
  __shared__ uint32_t count[4][kDigits], shared[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digits = 1 << p.bits;
  for (int d = threadIdx.x; d < 4 * kDigits; d += 256) (&count[0][0])[d] = 0;
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * kTile + wave * (kTile / 4) + lane;
  uint32_t key[ROUNDS], place[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = first + r * 64;
    key[r] = i < p.n ? p.key(i) : 0;
    place[r] = i < p.n ? (p.words ? uint32_t(i) : p.places[i]) : 0;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool in = first + r * 64 < p.n;
    const uint32_t d = p.digit(key[r]);
    uint64_t same = __ballot(in);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __ballot(d >> b & 1);
      same &= d >> b & 1 ? set : ~set;
    }
    const int leader = same ? __ffsll((unsigned long long)same) - 1 : 0;
    uint32_t before = 0;
    if (in && lane == leader) before = atomicAdd(&count[wave][d], uint32_t(__popcll(same)));
    rank[r] = __shfl(before, leader) + uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
  }
  __syncthreads();
  // counts of the waves become the first place of each one's digit
  const uint32_t *totals = p.counts + int64_t(digits) * p.tiles;
  uint32_t carry = 0;
  for (int d0 = 0; d0 < digits; d0 += 256) {
    const int d = d0 + int(threadIdx.x);
    uint32_t total;
    const uint32_t before = sum_before(d < digits ? totals[d] : 0, total, shared);
    if (d < digits) {
      uint32_t at = carry + before + p.counts[d * p.tiles + blockIdx.x];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t c = count[w][d];
        count[w][d] = at;
        at += c;
      }
    }
    carry += total;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r)
    if (first + r * 64 < p.n) {
      const uint32_t to = count[wave][p.digit(key[r])] + rank[r];
      p.keys_out[to] = key[r];
      p.places_out[to] = place[r];
    }
}

// ------------------------------------------------------------------ sums -----
// kPiece sorted places a piece.  What a word has inside one piece goes to its
// row of the gradient; what it has in a piece that it shares with the piece
// before (slot 0) or after it (slot 1, where it begins in this piece) goes to
// `part` [pieces][2][width], which k_join_words sums.
constexpr int kPiece = 64;

struct Sums {
  const uint32_t *keys, *places;
  int64_t n;
  uint32_t vocab;
  int width;
  float scale;
  float *part;
  int64_t pieces;
  __device__ uint32_t key(int64_t i) const { return i >= 0 && i < n ? keys[i] : vocab; }
};

template <typename T, int N>
__device__ inline void store_sum(T *row, const float (&s)[N], float scale) {
  Some<T, N> out;
#pragma unroll
  for (int e = 0; e < N; ++e) out.v[e] = T(s[e] * scale);
  out.store(row);
}

// A wave a piece and 64 N columns, eight rows of dy in flight.
template <typename T, int N>
__device__ inline void sum_piece(const Sums &a, const T *dy, int64_t lddy, T *dweight, int64_t piece, int c0) {
  constexpr int U = 8;
  const int lane = threadIdx.x & 63, c = c0 + lane * N;
  const int64_t first = piece * kPiece;
  const uint32_t key = a.key(first + lane);
  const uint32_t place = first + lane < a.n ? a.places[first + lane] : 0;
  const uint32_t before = piece ? a.keys[first - 1] : a.vocab, after = a.key(first + kPiece);
  const int count = __popcll(__ballot(key < a.vocab));  // sorted: the first ones
  if (count == 0) return;
  uint32_t next = __shfl_down(key, 1);  // of all lanes
  if (lane == 63) next = after;
  const uint64_t ends = __ballot(lane < count && (lane == count - 1 || next != key));
  bool open = before == __builtin_amdgcn_readfirstlane(key);  // the word began in an earlier piece
  const bool goes_on = count == kPiece && after == __builtin_amdgcn_readlane(key, 63);
  const bool in = c < a.width;
  float s[N];
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = 0.0f;
  for (int t0 = 0; t0 < count; t0 += U) {
    Some<T, N> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u, count - 1);
      const int64_t row = uint32_t(__builtin_amdgcn_readlane(place, t));
      if (in) v[u].load(dy + row * lddy + c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u;
      if (t >= count) break;
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] += float(v[u].v[e]);
      if (!(ends >> t & 1)) continue;
      if (in) {
        const bool on = t == kPiece - 1 && goes_on;
        if (open || on) {
          float *to = a.part + (piece * 2 + (open ? 0 : 1)) * a.width + c;
#pragma unroll
          for (int e = 0; e < N; ++e) to[e] = s[e];
        } else {
          store_sum<T, N>(dweight + int64_t(uint32_t(__builtin_amdgcn_readlane(key, t))) * a.width + c, s, a.scale);
        }
      }
      open = false;
#pragma unroll
      for (int e = 0; e < N; ++e) s[e] = 0.0f;
    }
  }
}

// The rows of words that no place has, kAbsent words a workgroup.
constexpr int kAbsent = 64;
template <typename T, int N>
__device__ inline void clear_absent(const Sums &a, T *dweight, int64_t first) {
  __shared__ int absent[kAbsent];
  const int64_t word = first + threadIdx.x;
  if (threadIdx.x < kAbsent) {
    bool found = true;
    if (word < a.vocab) {
      int64_t low = 0, high = a.n;  // the first place of a key not below the word
      while (low < high) {
        const int64_t mid = (low + high) >> 1;
        if (a.keys[mid] < word) low = mid + 1;
        else high = mid;
      }
      found = low < a.n && a.keys[low] == word;
    }
    absent[threadIdx.x] = !found;
  }
  __syncthreads();
  Some<T, N> zero;
#pragma unroll
  for (int e = 0; e < N; ++e) zero.v[e] = T(0.0f);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int w = wave; w < kAbsent; w += 4) {
    if (!absent[w]) continue;
    T *row = dweight + (first + w) * a.width;
    for (int c = lane * N; c < a.width; c += 64 * N) zero.store(row + c);
  }
}

template <typename T, int N>
__global__ __launch_bounds__(256) void k_word_sums(const Sums a, const T *dy, int64_t lddy, T *dweight, int groups,
                                                   int64_t sum_blocks) {
  if (int64_t(blockIdx.x) >= sum_blocks) {
    clear_absent<T, N>(a, dweight, (int64_t(blockIdx.x) - sum_blocks) * kAbsent);
    return;
  }
  const int64_t item = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t piece = item / groups;
  if (piece < a.pieces) sum_piece<T, N>(a, dy, lddy, dweight, piece, int(item % groups) * 64 * N);
}

// Words that go over the ends of pieces: the piece that a word begins in holds
// its first sum, the heads of the following pieces the others.  Up to kShort of
// them are summed by one wave, more by the workgroup's 16, each every 16th.
constexpr int kShort = 16, kJoin = 16;
template <typename T>
__global__ __launch_bounds__(1024) void k_join_words(const Sums a, T *dweight) {
  __shared__ float shared[kJoin][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = int(blockIdx.y) * 64 + lane;
  // how many pieces after p begin with the word that goes over p's end, 0 if none begins in p and does
  auto heads = [&](int64_t p, uint32_t &word) -> int64_t {
    if (p >= a.pieces) return 0;
    const int64_t end = (p + 1) * kPiece;
    word = a.key(end - 1);
    if (word >= a.vocab || a.key(end) != word) return 0;
    if (a.key(p * kPiece) == word && p > 0 && a.key(p * kPiece - 1) == word) return 0;
    const uint64_t same = __ballot(a.key(end + int64_t(lane) * kPiece) == word);
    if (~same) return __ffsll((unsigned long long)~same) - 1;
    int64_t low = p + 64, high = a.pieces - 1;  // the last piece whose first word it is
    while (low < high) {
      const int64_t mid = (low + high + 1) >> 1;
      if (a.key(mid * kPiece) == word) low = mid;
      else high = mid - 1;
    }
    return low - p;
  };
  auto head = [&](int64_t p) { return a.part[p * 2 * a.width + c]; };
  const int64_t p0 = int64_t(blockIdx.x) * kJoin;
  uint32_t word;
  const int64_t mine = heads(p0 + wave, word);
  if (mine > 0 && mine <= kShort && c < a.width) {
    const int64_t p = p0 + wave;
    float s = a.part[(p * 2 + 1) * a.width + c];
#pragma unroll 4
    for (int64_t i = 1; i <= mine; ++i) s += head(p + i);
    dweight[int64_t(word) * a.width + c] = T(s * a.scale);
  }
  __shared__ int64_t longer[kJoin];
  __shared__ uint32_t its[kJoin];
  if (lane == 0) {
    longer[wave] = mine > kShort ? mine : 0;
    its[wave] = word;
  }
  __syncthreads();
  for (int k = 0; k < kJoin; ++k) {
    const int64_t count = longer[k], p = p0 + k;
    if (!count) continue;
    float s = 0.0f;
    if (c < a.width) {
      if (wave == 0) s = a.part[(p * 2 + 1) * a.width + c];
#pragma unroll 8
      for (int64_t i = 1 + wave; i <= count; i += kJoin) s += head(p + i);
    }
    __syncthreads();
    shared[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < a.width) {
      for (int w = 1; w < kJoin; ++w) s += shared[w][lane];
      dweight[int64_t(its[k]) * a.width + c] = T(s * a.scale);
    }
  }
}

// ------------------------------------------------------------------ host -----
// How many elements of a matrix' rows can be moved at once, of most (16 bytes), 2 and 1.
template <typename T>
int at_once(const void *p, int64_t ld, int64_t cols) {
  for (int n : {16 / int(sizeof(T)), 2})
    if (n * sizeof(T) >= 4 && reinterpret_cast<uintptr_t>(p) % (n * sizeof(T)) == 0 && ld % n == 0 && cols % n == 0)
      return n;
  return 1;
}

template <typename T, typename Fn>
hipError_t by_count(int n, Fn fn) {
  if (n == 16 / int(sizeof(T))) return fn(std::integral_constant<int, 16 / int(sizeof(T))>());
  if (n == 2) return fn(std::integral_constant<int, 2>());
  return fn(std::integral_constant<int, 1>());
}

template <typename T>
hipError_t embed_forward_t(const lda_embed_args &a) {
  if (a.rows == 0) return hipSuccess;
  const int from = at_once<T>(a.weight, a.ld_weight, a.width), to = at_once<T>(a.y, a.ldy, a.width);
  return by_count<T>(from < to ? from : to, [&](auto count) {
    constexpr int N = decltype(count)::value;
    int shift = 0;
    while (shift < 8 && (N << shift) < a.width) ++shift;
    const int64_t each = int64_t(256 >> shift) * 4;
    k_embed<T, N><<<unsigned(ceil_div(a.rows, each)), 256, 0, static_cast<hipStream_t>(a.stream)>>>(
        a.words, a.rows, static_cast<const T *>(a.weight), a.ld_weight, a.width, a.vocab, a.scale, shift,
        static_cast<T *>(a.y), a.ldy);
    return hipGetLastError();
  });
}

struct Sorted {
  const uint32_t *keys, *places;
};

// The places 0 .. n - 1 by their words, in their order where these are equal.
hipError_t sort_words(const int32_t *words, int64_t n, int vocab, Arena &ws, bool dry, hipStream_t s, Sorted &out) {
  uint32_t *keys[2], *places[2];
  keys[0] = ws.take<uint32_t>(n);
  places[0] = ws.take<uint32_t>(n);
  out = Sorted{keys[0], places[0]};
  if (n <= kSmall) {
    if (dry || n == 0) return hipSuccess;
    int padded = 2;
    while (padded < n) padded <<= 1;
    k_sort_small<<<1, 1024, 0, s>>>(words, int(n), padded, uint32_t(vocab), keys[0], places[0]);
    return hipGetLastError();
  }
  keys[1] = ws.take<uint32_t>(n);
  places[1] = ws.take<uint32_t>(n);
  int bits = 1;
  while (uint32_t(vocab) >> bits) ++bits;
  const int passes = int(ceil_div(bits, kDigitBits)), each = int(ceil_div(bits, passes));
  SortPass p = {};
  p.n = n;
  p.vocab = uint32_t(vocab);
  p.bits = each;
  p.tiles = ceil_div(n, kTile);
  p.counts = ws.take<uint32_t>((p.tiles + 1) << each);
  for (int i = 0; i < passes; ++i) {
    p.words = i ? nullptr : words;
    p.keys = out.keys;
    p.places = out.places;
    p.keys_out = keys[(i + 1) & 1];
    p.places_out = places[(i + 1) & 1];
    p.shift = i * each;
    out = Sorted{p.keys_out, p.places_out};
    if (dry) continue;
    k_sort_count<<<unsigned(p.tiles), 256, 0, s>>>(p);
    OPS_TRY(hipGetLastError());
    k_sort_sums<<<1u << each, 256, 0, s>>>(p);
    OPS_TRY(hipGetLastError());
    k_sort_place<<<unsigned(p.tiles), 256, 0, s>>>(p);
    OPS_TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace

template <typename T>
hipError_t sum_by_word(const int32_t *words, int64_t n, const T *dy, int64_t lddy, int width, int vocab, float scale,
                       T *dweight, Arena &ws, bool dry, hipStream_t s) {
  Sorted order;
  OPS_TRY(sort_words(words, n, vocab, ws, dry, s, order));
  Sums a = {};
  a.keys = order.keys;
  a.places = order.places;
  a.n = n;
  a.vocab = uint32_t(vocab);
  a.width = width;
  a.scale = scale;
  a.pieces = ceil_div(n, kPiece);
  a.part = ws.take<float>(a.pieces * 2 * width);
  if (dry) return hipSuccess;
  const int from = at_once<T>(dy, lddy, width), to = at_once<T>(dweight, width, width);
  OPS_TRY(by_count<T>(from < to ? from : to, [&](auto count) {
    constexpr int N = decltype(count)::value;
    const int groups = int(ceil_div(width, 64 * N));
    const int64_t sums = ceil_div(a.pieces * groups, 4);
    k_word_sums<T, N><<<unsigned(sums + ceil_div(vocab, kAbsent)), 256, 0, s>>>(a, dy, lddy, dweight, groups, sums);
    return hipGetLastError();
  }));
  if (a.pieces <= 1) return hipSuccess;
  k_join_words<T><<<dim3(unsigned(ceil_div(a.pieces, kJoin)), unsigned(ceil_div(width, 64))), 1024, 0, s>>>(a, dweight);
  return hipGetLastError();
}

template hipError_t sum_by_word<float>(const int32_t *, int64_t, const float *, int64_t, int, int, float, float *,
                                       Arena &, bool, hipStream_t);

namespace {

template <typename T>
hipError_t embed_backward_t(const lda_embed_args &a, Arena &ws, bool dry) {
  return sum_by_word<T>(a.words, a.rows, static_cast<const T *>(a.dy), a.lddy, a.width, a.vocab, a.scale,
                        static_cast<T *>(a.dweight), ws, dry, static_cast<hipStream_t>(a.stream));
}

}  // namespace

hipError_t embed_forward(const lda_embed_args &a) {
  switch (a.dtype) {
    case LDA_F32: return embed_forward_t<float>(a);
    case LDA_BF16: return embed_forward_t<bf16>(a);
    default: return embed_forward_t<f16>(a);
  }
}

hipError_t embed_backward(const lda_embed_args &a, Arena &ws, bool dry) {
  switch (a.dtype) {
    case LDA_F32: return embed_backward_t<float>(a, ws, dry);
    case LDA_BF16: return embed_backward_t<bf16>(a, ws, dry);
    default: return embed_backward_t<f16>(a, ws, dry);
  }
}

}  // namespace ops
}  // namespace lda
