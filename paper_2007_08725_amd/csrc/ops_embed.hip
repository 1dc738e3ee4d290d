// Word embedding and its gradient (include/lda_ops.h).
//
// The forward pass copies rows of the table.  The backward pass sorts the rows
// of dy by word, so that a word's gradient is a sum over neighbours in the
// order, and sums pieces of a fixed number of sorted rows: a word that is a
// tenth of the corpus then costs no more than its rows, and no sum depends on
// the order in which workgroups run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ops_internal.h"

#pragma clang fp contract(fast)

namespace lda {
namespace ops {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

// The columns of a row that a lane moves at once: 16 bytes, wherever they begin
// (global memory takes vectors at any address).  Where a row is no multiple of
// them its last lane takes the last 16 bytes of the row, some of which another
// lane has too: both compute the same.  Rows shorter than that (Narrow) element
// by element.
template <typename T>
constexpr int kMany = 16 / int(sizeof(T));
template <typename T, bool Narrow>
struct Many {
  static constexpr int N = kMany<T>;
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  T v[N];
  static __device__ int first(int lane, int cols) { return Narrow ? 0 : min(lane * N, cols - N); }
  __device__ void clear() {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = T(0.0f);
  }
  __device__ void load(const T *p, int cols) {
    if constexpr (Narrow) {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < cols ? p[e] : T(0.0f);
    } else {
      const vec w = *reinterpret_cast<const vec *>(p);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = w[e];
    }
  }
  template <bool Past = false>
  __device__ void store(T *p, int cols) const {
    if constexpr (Narrow) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < cols) p[e] = v[e];
    } else {
      vec w;
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = v[e];
      if constexpr (Past) __builtin_nontemporal_store(w, reinterpret_cast<vec *>(p));
      else *reinterpret_cast<vec *>(p) = w;
    }
  }
};

// -------------------------------------------------------------- forward -----
// 2^shift lanes a row (a workgroup has 256 >> shift rows at a time), four rows
// of each lane in flight.
//
// Bound by its bytes: 65536 words x 1024 of bf16 from a table of 141000 rows 37 us
// = 4.4 TB/s of y and the rows that are named, 1048576 x 512 of f16 281 us = 4.0.
// Rows that do not lie on a grid of 16 bytes take longer: 50000 x 256 from 2000 rows in
// single precision 11.0 us a call, x 257 15.2.
//
// Results that are larger than the last cache (256 MB) are stored past it, so
// that it keeps the table and dy: both passes over 1048576 words x 512 of f16
// 673 -> 636 us.  Smaller ones are left in it for who reads them (both passes
// over 50000 x 257 in single precision, when they took 63 us: past it 77).
template <typename T, bool Narrow, bool Past>
__global__ __launch_bounds__(256) void k_embed(const int32_t *words, int64_t rows, const T *weight, int64_t ldw,
                                               int width, int vocab, float scale, int shift, T *y, int64_t ldy) {
  constexpr int U = 4, N = kMany<T>;
  const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), each = 256 >> shift;
  const int64_t first = int64_t(blockIdx.x) * each * U + (threadIdx.x >> shift);
  int word[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = first + u * each;
    word[u] = i < rows ? words[i] : -1;
  }
  for (int i = lane; i * N < width; i += lanes) {
    const int c = Many<T, Narrow>::first(i, width);
    Many<T, Narrow> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (word[u] >= 0 && word[u] < vocab) v[u].load(weight + int64_t(word[u]) * ldw + c, width);
      else v[u].clear();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = first + u * each;
      if (row >= rows) break;
#pragma unroll
      for (int e = 0; e < N; ++e) v[u].v[e] = T(float(v[u].v[e]) * scale);
      v[u].template store<Past>(y + row * ldy + c, width);
    }
  }
}

// ------------------------------------------------------------------ sort -----
// The gradient's rows are set to zero by further workgroups of the sort's
// launches, which leave most of the machine idle, each launch a part of them
// (65536 words and a gradient of 141000 x 1024 of bf16: 289 MB beside 45 us of
// sorting); rows of words that there are get their sums afterwards.  Past the last
// cache, where the zeros would push out what is summed next (175 us -> 155 for
// both passes).
//
// Vectors and words of memory that is aligned to an element of 16 bits.
typedef uint32_t fill_word __attribute__((aligned(2)));
typedef uint32_t fill_words __attribute__((ext_vector_type(4), aligned(2)));
struct Fill {
  fill_word *p;
  int64_t words, bytes;  // whole words of 32 bits; the bytes after them, in the last launch's last workgroup
  int64_t from, to;      // of this launch, words
};
constexpr int kFillWords = 16384;  // of a workgroup: 64 KiB

__device__ inline void fill_zero(const Fill &f, int64_t part) {
  const int64_t first = f.from + part * kFillWords, end = first + kFillWords < f.to ? first + kFillWords : f.to;
  int64_t i = first + int64_t(threadIdx.x) * 4;
  for (; i + 4 <= end; i += int64_t(blockDim.x) * 4)
    __builtin_nontemporal_store(fill_words{0, 0, 0, 0}, reinterpret_cast<fill_words *>(f.p + i));
  for (; i < end; ++i) f.p[i] = 0;
  if (end == f.words && threadIdx.x < f.bytes) reinterpret_cast<uint8_t *>(f.p + f.words)[threadIdx.x] = 0;
}
__host__ __device__ inline int64_t fill_parts(const Fill &f) {
  return (f.to - f.from + kFillWords - 1) / kFillWords + (f.to == f.words && f.from == f.to && f.bytes ? 1 : 0);
}

// Keys are the words, and `vocab` for places of no word, which so come last.
__device__ inline uint32_t key_of(int32_t word, uint32_t vocab) {
  return uint32_t(word) < vocab ? uint32_t(word) : vocab;
}

// The lanes of a wave whose place is `in` and has the same digit, by a ballot a bit.
__device__ inline uint64_t same_digit(uint32_t digit, int bits, bool in) {
  uint64_t same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}

// A place's rank among those of its digit in its wave: what the wave had of them
// already (count, which goes on), and the lanes before it.
__device__ inline uint32_t rank_in_wave(uint32_t digit, int bits, bool in, int lane, uint32_t *count) {
  const uint64_t same = same_digit(digit, bits, in);
  const int leader = same ? __ffsll((unsigned long long)same) - 1 : 0;
  uint32_t before = 0;
  if (in && lane == leader) before = atomicAdd(count + digit, uint32_t(__popcll(same)));
  return __shfl(before, leader) + uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
}

// Up to kSmall places in one workgroup, which has them in its registers and moves
// them through LDS, a radix sort from the lowest 6 bits on: 8192 words of a
// vocabulary of 102000 (three passes) 24 us, 4096 of one of 2000 (two) 11; a
// bitonic network took 75 and 37.
constexpr int kSmall = 8192, kSmallBits = 6;
__global__ __launch_bounds__(1024) void k_sort_small(const int32_t *words, int n, int passes, uint32_t vocab,
                                                     uint32_t *keys, uint32_t *places, const Fill fill) {
  constexpr int ROUNDS = kSmall / 1024, DIGITS = 1 << kSmallBits;
  __shared__ uint32_t all_keys[kSmall], count[16][DIGITS], sums[16];
  __shared__ uint16_t all_places[kSmall];
  if (blockIdx.x > 0) {
    fill_zero(fill, int64_t(blockIdx.x) - 1);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rounds = (n + 1023) / 1024;
  const int first = wave * rounds * 64 + lane;
  uint32_t key[ROUNDS], place[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * 64;
    key[r] = r < rounds && i < n ? key_of(words[i], vocab) : 0;
    place[r] = i;
  }
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * kSmallBits;
    (&count[0][0])[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (r >= rounds) break;
      rank[r] = rank_in_wave(key[r] >> shift & (DIGITS - 1), kSmallBits, first + r * 64 < n, lane, count[wave]);
    }
    __syncthreads();
    // thread d * 16 + w: the first place of digit d of wave w
    const int d = threadIdx.x >> 4, w = threadIdx.x & 15;
    const uint32_t mine = count[w][d];
    uint32_t upto = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const uint32_t other = __shfl_up(upto, x);
      if (lane >= x) upto += other;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (int x = 0; x < wave; ++x) at += sums[x];
    count[w][d] = at;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (r >= rounds || first + r * 64 >= n) continue;
      const uint32_t to = count[wave][key[r] >> shift & (DIGITS - 1)] + rank[r];
      all_keys[to] = key[r];
      all_places[to] = uint16_t(place[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (r >= rounds || first + r * 64 >= n) continue;
      key[r] = all_keys[first + r * 64];
      place[r] = all_places[first + r * 64];
    }
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    if (r >= rounds || first + r * 64 >= n) continue;
    keys[first + r * 64] = key[r];
    places[first + r * 64] = place[r];
  }
}

// More: a radix sort from the lowest digit of up to kDigitBits bits on, three
// launches a digit: counts of each tile, their sums before each tile, and the
// tile's places moved to where they belong, in their order.  1048576 words of
// 102000, two digits: 60 us in six launches, bound by their chains of loads,
// ballots and barriers (their bytes alone take 12).
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kTile = 1024;
struct SortPass {
  const int32_t *words;  // of the first pass: keys from the words, places 0, 1, ..
  const uint32_t *keys, *places;
  uint32_t *keys_out, *places_out;
  int64_t n;
  uint32_t vocab;
  int shift, bits;
  // places of a tile, a multiple of 256: few where there are few places, so that they spread over the CUs (16384: 256
  // instead of 1024 49 us for both passes instead of 56), up to kTile (1048576 with 512: 614 us, with 1024 601)
  int tile;
  int64_t tiles;
  uint32_t *counts;  // [tiles][digits], then the digits' totals
  __device__ uint32_t key(int64_t i) const { return words ? key_of(words[i], vocab) : keys[i]; }
  __device__ uint32_t digit(uint32_t key) const { return key >> shift & ((1u << bits) - 1); }
};

__global__ __launch_bounds__(256) void k_sort_count(const SortPass p, const Fill fill) {
  __shared__ uint32_t count[kDigits];
  if (int64_t(blockIdx.x) >= p.tiles) {
    fill_zero(fill, int64_t(blockIdx.x) - p.tiles);
    return;
  }
  const int digits = 1 << p.bits;
  for (int d = threadIdx.x; d < digits; d += 256) count[d] = 0;
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * p.tile;
  for (int i = threadIdx.x; i < p.tile; i += 256)
    if (first + i < p.n) atomicAdd(&count[p.digit(p.key(first + i))], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += 256) p.counts[int64_t(blockIdx.x) * digits + d] = count[d];
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

// The digits' counts become the sums of the tiles before.  A workgroup takes
// kSide digits (64 bytes of a tile's counts), and kLong tiles at a time in
// kLong / kDeep threads a digit, each with kDeep neighbouring tiles.
constexpr int kSide = 16, kDeep = 16, kLong = 1024 / kSide * kDeep;
__global__ __launch_bounds__(1024) void k_sort_sums(const SortPass p, const Fill fill) {
  __shared__ uint32_t shared[16][kSide];
  const int digits = 1 << p.bits, groups = (digits + kSide - 1) / kSide;
  if (int(blockIdx.x) >= groups) {
    fill_zero(fill, int64_t(blockIdx.x) - groups);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int d = int(blockIdx.x) * kSide + (lane & (kSide - 1)), row = int(threadIdx.x) / kSide;
  const bool in = d < digits;
  uint32_t carry = 0;
  for (int64_t t0 = 0; t0 < p.tiles; t0 += kLong) {
    const int64_t first = t0 + row * kDeep;
    uint32_t v[kDeep], sum = 0;
#pragma unroll
    for (int i = 0; i < kDeep; ++i) v[i] = in && first + i < p.tiles ? p.counts[(first + i) * digits + d] : 0;
#pragma unroll
    for (int i = 0; i < kDeep; ++i) sum += v[i];
    // over the wave's four rows, then over the waves
    uint32_t upto = sum;
#pragma unroll
    for (int x = kSide; x < 64; x <<= 1) {
      const uint32_t other = __shfl_up(upto, x);
      if (lane >= x) upto += other;
    }
    __syncthreads();
    if (lane >= 64 - kSide) shared[wave][lane & (kSide - 1)] = upto;
    __syncthreads();
    uint32_t before = carry + upto - sum;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      const uint32_t all = shared[w][lane & (kSide - 1)];
      if (w < wave) before += all;
      carry += all;
    }
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      if (in && first + i < p.tiles) p.counts[(first + i) * digits + d] = before;
      before += v[i];
    }
  }
  if (row == 0 && in) p.counts[p.tiles * digits + d] = carry;
}

// Each wave takes a quarter of the tile, 64 places at a time.
__global__ __launch_bounds__(256) void k_sort_place(const SortPass p, const Fill fill) {
  constexpr int ROUNDS = kTile / 256;
  __shared__ uint32_t count[4][kDigits], shared[4];
  if (int64_t(blockIdx.x) >= p.tiles) {
    fill_zero(fill, int64_t(blockIdx.x) - p.tiles);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digits = 1 << p.bits;
  for (int d = threadIdx.x; d < 4 * digits; d += 256) count[d / digits][d % digits] = 0;
  __syncthreads();
  const int64_t first = int64_t(blockIdx.x) * p.tile + wave * (p.tile / 4) + lane;
  const int64_t end = min(p.n, first - lane + p.tile / 4);
  uint32_t key[ROUNDS], place[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = first + r * 64;
    key[r] = i < end ? p.key(i) : 0;
    place[r] = i < end ? (p.words ? uint32_t(i) : p.places[i]) : 0;
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    if (r * 256 >= p.tile) break;
    rank[r] = rank_in_wave(p.digit(key[r]), p.bits, first + r * 64 < end, lane, count[wave]);
  }
  __syncthreads();
  // counts of the waves become the first place of each one's digit
  const uint32_t *totals = p.counts + int64_t(digits) * p.tiles, *mine = p.counts + int64_t(blockIdx.x) * digits;
  uint32_t carry = 0;
  for (int d0 = 0; d0 < digits; d0 += 256) {
    const int d = d0 + int(threadIdx.x);
    uint32_t total;
    const uint32_t before = sum_before(d < digits ? totals[d] : 0, total, shared);
    if (d < digits) {
      uint32_t at = carry + before + mine[d];
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
    if (first + r * 64 < end) {
      const uint32_t to = count[wave][p.digit(key[r])] + rank[r];
      p.keys_out[to] = key[r];
      p.places_out[to] = place[r];
    }
}

// ------------------------------------------------------------------ sums -----
// `each` sorted places a piece, a power of two.  What a word has inside one
// piece goes to its row of the gradient; what it has in a piece that it shares
// with the piece before (slot 0) or after it (slot 1, where it begins in this
// piece) goes to `part` [pieces][2][width], which k_join_words sums.
//
// Sums are kept in 32 bits for 16-bit types, whose own rounding is 2^13 or 2^16
// times theirs, and in 64 for single precision: added there in 32 bits, one after
// another, a word of 5,000 rows is off by 5.6 times its result's rounding and one of
// 105,000 by 8.5, sums that cancel by any part of themselves.  It costs both passes
// over 50000 x 257 of 2000 words 58.6 -> 59.7 us, the backward pass over 1048576 x 256
// of 102000 319 -> 333.
template <typename T>
using Total = std::conditional_t<sizeof(T) == 4, double, float>;
template <typename T>
struct Sums {
  const uint32_t *keys, *places;
  int64_t n;
  uint32_t vocab;
  int width;
  float scale;
  Total<T> *part;
  int64_t pieces;
  int each;
  __device__ uint32_t key(int64_t i) const { return i >= 0 && i < n ? keys[i] : vocab; }
};

// A wave a piece and 64 kMany columns, eight rows of dy in flight.  Bound by dy's
// bytes, in rows that lie anywhere: 65536 x 1024 of bf16 38 us = 3.5 TB/s, 1048576
// x 512 of f16 247 us = 4.3.
template <typename T, bool Narrow>
__global__ __launch_bounds__(256) void k_word_sums(const Sums<T> a, const T *dy, int64_t lddy, T *dweight, int groups) {
  constexpr int U = 4, N = kMany<T>;
  const int64_t item = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t piece = item / groups;
  if (piece >= a.pieces) return;
  const int lane = threadIdx.x & 63, mine = int(item % groups) * 64 + lane;
  const bool in = mine * N < a.width;
  const int c = Many<T, Narrow>::first(mine, a.width);
  const int64_t begin = piece * a.each;
  bool open = false;  // the word began in an earlier piece
  Total<T> s[N];
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = 0;
  const int span = min(64, a.each);  // places at a time
  for (int64_t first = begin; first < begin + a.each; first += span) {
    const uint32_t key = lane < span ? a.key(first + lane) : a.vocab;
    const uint32_t place = lane < span && first + lane < a.n ? a.places[first + lane] : 0;
    const uint32_t after = a.key(first + span);
    uint32_t next = __shfl_down(key, 1);  // of all lanes
    if (lane == span - 1) next = after;
    const int count = __popcll(__ballot(key < a.vocab));  // sorted: the first ones
    if (count == 0) return;
    if (first == begin && begin > 0) open = a.keys[begin - 1] == __builtin_amdgcn_readfirstlane(key);
    // places after which a sum ends: with its word, or with the piece
    const bool last = first + span == begin + a.each;
    const uint64_t ends = __ballot(lane < count && (next != key || (last && lane == span - 1)));
    const bool goes_on = last && count == span && after == __builtin_amdgcn_readlane(key, span - 1);
    auto load = [&](Many<T, Narrow>(&v)[U], int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t row = uint32_t(__builtin_amdgcn_readlane(place, min(t0 + u, count - 1)));
        v[u].load(dy + row * lddy + c, a.width);
      }
    };
    auto add = [&](const Many<T, Narrow>(&v)[U], int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + u;
        if (t >= count) break;
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] += Total<T>(v[u].v[e]);
        if (!(ends >> t & 1)) continue;
        if (open || (goes_on && t == span - 1)) {
          Total<T> *to = a.part + (piece * 2 + (open ? 0 : 1)) * a.width + c;
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (in && (!Narrow || e < a.width)) to[e] = s[e];
        } else if (in) {
          Many<T, Narrow> out;
#pragma unroll
          for (int e = 0; e < N; ++e) out.v[e] = T(s[e] * a.scale);
          out.store(dweight + int64_t(uint32_t(__builtin_amdgcn_readlane(key, t))) * a.width + c, a.width);
        }
        open = false;
#pragma unroll
        for (int e = 0; e < N; ++e) s[e] = 0;
      }
    };
    // the next rows are asked for before this ones' sums are stored: a wave waits for what it asked for in its order
    Many<T, Narrow> even[U], odd[U];
    load(even, 0);
    for (int t0 = 0; t0 < count; t0 += 2 * U) {
      load(odd, t0 + U);
      add(even, t0);
      load(even, t0 + 2 * U);
      add(odd, t0 + U);
    }
  }
}

// Words that go over the ends of pieces: the piece that a word begins in holds
// its first sum, the heads of the following pieces the others.  A workgroup looks
// at kJoin pieces; up to kShort heads are summed by one wave, more by all of
// them, each every kJoin-th.  8 to 26 us, a chain of four to six loads.  A lane has 16
// bytes of sums, 4 or 2 columns.
constexpr int kShort = 16, kJoin = 16;
template <typename T>
__global__ __launch_bounds__(1024) void k_join_words(const Sums<T> a, T *dweight) {
  constexpr int U = 8, C = 16 / int(sizeof(Total<T>));
  __shared__ Total<T> shared[kJoin][64 * C];
  __shared__ int64_t longer[kJoin];
  __shared__ uint32_t its[kJoin];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int mine_c = (int(blockIdx.y) * 64 + lane) * C;
  const int64_t p0 = int64_t(blockIdx.x) * kJoin, p = p0 + wave, end = (p + 1) * a.each;
  // how many pieces after p begin with the word that begins in p and goes over its end
  uint32_t word = a.vocab;
  int64_t mine = 0;
  if (p < a.pieces) {
    // the last place, the next one, the first one and the one before it
    const uint32_t at = a.key(lane < 2 ? end - 1 + lane : p * a.each + 2 - lane);
    word = __builtin_amdgcn_readlane(at, 0);
    const bool over = word < a.vocab && __builtin_amdgcn_readlane(at, 1) == word;
    const bool before = p > 0 && __builtin_amdgcn_readlane(at, 2) == word && __builtin_amdgcn_readlane(at, 3) == word;
    if (over && !before) {
      int64_t low = p + 1;  // the last piece that is known to begin with it
      auto ahead = [&](int64_t step) {
        const uint64_t same = __ballot(a.key((low + (lane + 1) * step) * a.each) == word);
        const int count = ~same ? __ffsll((unsigned long long)~same) - 1 : 64;
        low += count * step;
        return count == 64;
      };
      if (ahead(1)) {
        while (ahead(64)) {}
        ahead(1);
      }
      mine = low - p;
    }
  }
  const bool narrow = a.width < C;
  const int c = narrow ? 0 : min(mine_c, a.width - C);
  typedef Total<T> some __attribute__((ext_vector_type(C), aligned(sizeof(Total<T>))));
  // what k_word_sums left of piece q in `slot`
  auto left = [&](int64_t q, int slot) {
    const Total<T> *from = a.part + (q * 2 + slot) * a.width + c;
    if (!narrow) return *reinterpret_cast<const some *>(from);
    some s = {};
#pragma unroll
    for (int e = 0; e < C - 1; ++e) s[e] = e < a.width ? from[e] : 0;
    return s;
  };
  // the heads after piece q, from the first-th to the count-th, every step-th: eight on their way at a time
  auto heads = [&](int64_t q, int64_t first, int64_t count, int step, some s) {
    for (int64_t i = first; i <= count; i += U * step) {
      some v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = left(q + (i + u * step <= count ? i + u * step : i), 0);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * step <= count) s += v[u];
    }
    return s;
  };
  auto store = [&](some s, uint32_t to) {
#pragma unroll
    for (int e = 0; e < C; ++e)
      if (c + e < a.width) dweight[int64_t(to) * a.width + c + e] = T(s[e] * a.scale);
  };
  if (mine > 0 && mine <= kShort && mine_c < a.width) store(heads(p, 1, mine, 1, left(p, 1)), word);
  if (lane == 0) {
    longer[wave] = mine > kShort ? mine : 0;
    its[wave] = word;
  }
  __syncthreads();
  for (int k = 0; k < kJoin; ++k) {
    const int64_t count = longer[k], q = p0 + k;
    if (!count) continue;
    some s = {};
    if (mine_c < a.width) s = heads(q, 1 + wave, count, kJoin, wave == 0 ? left(q, 1) : s);
    __syncthreads();
    *reinterpret_cast<some *>(&shared[wave][lane * C]) = s;
    __syncthreads();
    if (wave == 0 && mine_c < a.width) {
      for (int w = 1; w < kJoin; ++w) s += *reinterpret_cast<const some *>(&shared[w][lane * C]);
      store(s, its[k]);
    }
  }
}

// ------------------------------------------------------------------ host -----
template <typename T>
hipError_t embed_forward_t(const lda_embed_args &a) {
  if (a.rows == 0) return hipSuccess;
  // 16 lanes a row if it has as many, more as long as no more of them are idle at its end
  int shift = 0;
  int64_t least = INT64_MAX;
  for (int i = 0; i <= 8; ++i) {
    const int64_t padded = round_up(a.width, int64_t(kMany<T>) << i);
    if (i > 4 && padded > least) break;
    shift = i;
    least = padded;
    if (padded == int64_t(kMany<T>) << i) break;
  }
  const int64_t each = int64_t(256 >> shift) * 4;
  const bool past = a.rows * a.width * int64_t(sizeof(T)) >= int64_t(256) << 20;
  auto kernel = a.width < kMany<T> ? k_embed<T, true, false> : past ? k_embed<T, false, true> : k_embed<T, false, false>;
  kernel<<<unsigned(ceil_div(a.rows, each)), 256, 0, static_cast<hipStream_t>(a.stream)>>>(
      a.words, a.rows, static_cast<const T *>(a.weight), a.ld_weight, a.width, a.vocab, a.scale, shift,
      static_cast<T *>(a.y), a.ldy);
  return hipGetLastError();
}

struct Sorted {
  const uint32_t *keys, *places;
};

// A launch's part of `all`, of which the next `launches` ones have equal shares.
Fill share(Fill &all, int launches) {
  Fill now = all;
  now.to = launches <= 1 ? all.words : all.from + round_up(ceil_div(all.words - all.from, launches), kFillWords);
  if (now.to > all.words) now.to = all.words;
  all.from = now.to;
  return now;
}

// The places 0 .. n - 1 by their words, in their order where these are equal; and
// `fill` set to zero.
hipError_t sort_words(const int32_t *words, int64_t n, int vocab, Fill fill, Arena &ws, bool dry, hipStream_t s,
                      Sorted &out) {
  uint32_t *keys[2], *places[2];
  keys[0] = ws.take<uint32_t>(n);
  places[0] = ws.take<uint32_t>(n);
  out = Sorted{keys[0], places[0]};
  int bits = 1;
  while (uint32_t(vocab) >> bits) ++bits;
  if (n <= kSmall) {
    if (dry) return hipSuccess;
    const Fill all = share(fill, 1);
    k_sort_small<<<unsigned(1 + fill_parts(all)), 1024, 0, s>>>(
        words, int(n), int(ceil_div(bits, kSmallBits)), uint32_t(vocab), keys[0], places[0], all);
    return hipGetLastError();
  }
  keys[1] = ws.take<uint32_t>(n);
  places[1] = ws.take<uint32_t>(n);
  const int passes = int(ceil_div(bits, kDigitBits)), each = int(ceil_div(bits, passes));
  SortPass p = {};
  p.n = n;
  p.vocab = uint32_t(vocab);
  p.bits = each;
  p.tile = n < int64_t(1) << 17 ? kTile / 4 : n < int64_t(1) << 19 ? kTile / 2 : kTile;
  p.tiles = ceil_div(n, p.tile);
  p.counts = ws.take<uint32_t>((p.tiles + 1) << each);
  int launches = 3 * passes;
  for (int i = 0; i < passes; ++i) {
    p.words = i ? nullptr : words;
    p.keys = out.keys;
    p.places = out.places;
    p.keys_out = keys[(i + 1) & 1];
    p.places_out = places[(i + 1) & 1];
    p.shift = i * each;
    out = Sorted{p.keys_out, p.places_out};
    if (dry) continue;
    Fill part = share(fill, launches--);
    k_sort_count<<<unsigned(p.tiles + fill_parts(part)), 256, 0, s>>>(p, part);
    OPS_TRY(hipGetLastError());
    part = share(fill, launches--);
    k_sort_sums<<<unsigned(ceil_div(int64_t(1) << each, kSide) + fill_parts(part)), 1024, 0, s>>>(p, part);
    OPS_TRY(hipGetLastError());
    part = share(fill, launches--);
    k_sort_place<<<unsigned(p.tiles + fill_parts(part)), 256, 0, s>>>(p, part);
    OPS_TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace

template <typename T>
hipError_t sum_by_word(const int32_t *words, int64_t n, const T *dy, int64_t lddy, int width, int vocab, float scale,
                       T *dweight, Arena &ws, bool dry, hipStream_t s) {
  Fill fill = {};
  fill.p = reinterpret_cast<fill_word *>(dweight);
  const int64_t bytes = int64_t(vocab) * width * int64_t(sizeof(T));
  fill.words = bytes / 4;
  fill.bytes = bytes % 4;
  Sorted order;
  OPS_TRY(sort_words(words, n, vocab, fill, ws, dry, s, order));
  Sums<T> a = {};
  a.keys = order.keys;
  a.places = order.places;
  a.n = n;
  a.vocab = uint32_t(vocab);
  a.width = width;
  a.scale = scale;
  // short pieces where there are few waves otherwise (16384 words x 256 of bf16: of 64 72 us, of 16 54 for both
  // passes), longer ones where there are enough: less to join (1048576 x 512 of f16: of 128 743, of 256 686)
  const int groups = int(ceil_div(width, 64 * kMany<T>));
  a.each = 16;
  while (a.each < 512 && ceil_div(n, 2 * a.each) * groups >= 3000) a.each *= 2;
  a.pieces = ceil_div(n, a.each);
  a.part = ws.take<Total<T>>(a.pieces * 2 * width);
  if (dry || n == 0) return hipSuccess;
  auto kernel = width < kMany<T> ? k_word_sums<T, true> : k_word_sums<T, false>;
  kernel<<<unsigned(ceil_div(a.pieces * groups, 4)), 256, 0, s>>>(a, dy, lddy, dweight, groups);
  OPS_TRY(hipGetLastError());
  if (a.pieces <= 1) return hipSuccess;
  const int64_t strips = ceil_div(width, 64 * 16 / int64_t(sizeof(Total<T>)));
  k_join_words<T><<<dim3(unsigned(ceil_div(a.pieces, kJoin)), unsigned(strips)), 1024, 0, s>>>(a, dweight);
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
