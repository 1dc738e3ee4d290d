// Matrix products of the word-model operators (include/lda_ops.h): the gated
// layer, the softmax cross entropy and distillation, forward and backward.
//
// Every product is C[m][n] = sum_k L[m][k] R[n][k] on the matrix units, either
// operand as it lies in memory or transposed; what is done with C (activation,
// softmax statistics, gradient of the logits, store) is the epilogue of the
// kernel that computes it, while C is still in registers.  Sums are in 32 bits.
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
// r = 0..3 (of a fragment of R's rows: Order): four neighbours along the
// contiguous axis of C.
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
__device__ inline f32x4 mma_one(u32x4 r, u32x4 l, int e, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, r)[e], __builtin_bit_cast(f32x4, l)[e], c, 0, 0,
                                              0);
}
template <>
__device__ inline f32x4 mma<float>(u32x4 r, u32x4 l, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = mma_one(r, l, e, c);
  return c;
}

// Operands.  A step of the product takes 64 bytes of k of every row (kStep
// elements), in 16-byte chunks (kChunk elements).  An operand lies in memory
// either with k contiguous ("rows") or with its rows contiguous ("columns":
// the transposed matrix, element (row, k) at p[k * ld + row]); neither is
// copied for the other, LDS is read transposed.  `base` gives the address of
// the chunk that a lane loads in step 0, `ahead` how far on it lies in a later
// step, `in` whether its chunk of a
// step lies inside k.  Rows past the end
// repeat the last one (or chunk): their products go nowhere, and no read
// leaves the matrix.
template <typename T>
constexpr int kChunk = 16 / int(sizeof(T));
template <typename T>
constexpr int kStep = 64 / int(sizeof(T));

template <typename T>
struct Rows {
  static constexpr bool kContiguous = true;
  const T *p;
  int64_t ld;
  int rows, k;
  __device__ int64_t ahead(int step) const { return int64_t(step) * 64; }
  __device__ const char *base(int row, int k0) const {
    return reinterpret_cast<const char *>(p + int64_t(min(row, rows - 1)) * ld + k0);
  }
  __device__ bool in(int step, int k0) const { return step * kStep<T> + k0 < k; }
};

template <typename T>
struct Columns {
  static constexpr bool kContiguous = false;
  const T *p;
  int64_t ld;
  int rows, k;
  __device__ int64_t ahead(int step) const { return step * 64 * ld; }
  __device__ const char *base(int row, int k0) const {
    return reinterpret_cast<const char *>(p + int64_t(k0) * ld + min(row, (rows - 1) / kChunk<T> * kChunk<T>));
  }
  __device__ bool in(int step, int k0) const { return step * kStep<T> + k0 < k; }
};

// The rows of w_gate and w_value in turns of four: row n of the pair is row
// (n / 8) * 4 + n % 4 of w_gate where n & 4 is 0, else of w_value.  A lane that
// holds four neighbours of a then holds the same four of b in its next
// fragment.
__device__ inline int pair_row(int n) { return (n >> 3) * 4 + (n & 3); }

template <typename T>
struct PairRows {
  static constexpr bool kContiguous = true;
  const T *gate, *value;
  int64_t ld_gate, ld_value;
  int hidden, k;
  __device__ int64_t ahead(int step) const { return int64_t(step) * 64; }
  __device__ const char *base(int n, int k0) const {
    const int64_t f = min(pair_row(n), hidden - 1);
    return reinterpret_cast<const char *>((n & 4 ? value + f * ld_value : gate + f * ld_gate) + k0);
  }
  __device__ bool in(int step, int k0) const { return step * kStep<T> + k0 < k; }
};

// The pair as an operand of dx, whose k runs over the pair's rows.
template <typename T>
struct PairColumns {
  static constexpr bool kContiguous = false;
  const T *gate, *value;
  int64_t ld;  // of both
  int width, hidden;
  __device__ int64_t ahead(int step) const { return step * 32 * ld; }
  __device__ const char *base(int row, int k0) const {
    return reinterpret_cast<const char *>((k0 & 4 ? value : gate) + int64_t(pair_row(k0)) * ld +
                                          min(row, (width - 1) / kChunk<T> * kChunk<T>));
  }
  __device__ bool in(int step, int k0) const { return pair_row(step * kStep<T> + k0) < hidden; }
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
  // steps of k in all and of one split, both even (past the end of k all is
  // zero), and the splits (none is empty)
  int steps, split, splits;
};

// what a lane whose chunk lies past the end of k reads instead
__device__ const u32x4 kZeroChunk = {0, 0, 0, 0};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) uint32_t lds_u32;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Tile order: the tiles are cut into eight runs, one for each accelerator die
// (workgroups go to the dies in turn), and a run walks groups of eight tile
// rows column by column, so that the tiles a die works on at one time share
// their operands in its L2.
__device__ inline void tile_at(const Grid &g, int t, int &mt, int &nt) {
  const int group = 8 * g.ntiles, first = t / group * 8;
  const int high = min(8, g.mtiles - first), in = t % group;
  mt = first + in % high;
  nt = in / high;
}

// An operand's part of a stage in LDS, B rows: B/16 loads of 1 KiB, dealt to the
// waves in turns.
//
// k contiguous: 64 bytes a row; chunk c of row r lies at place c ^ chunk_turn(r).
//
// Rows contiguous: kStep lines of B elements, in slots of 16 rows, a slot in
// 16-byte parts.  Four 16-bit lines of a slot are what one transposing read of
// 16 lanes takes (8 bytes each: lane q reads line q / 4, four rows, and gets
// one row of the four lines); in single precision a line's slot is one read.
// Slots and parts of a line are permuted by the line's number.
//
// The permutations spread what is read together over the banks, for the 16
// neighbouring rows of a fragment of L as for the four times four rows that a
// fragment of R may take (Order).
__device__ inline int chunk_turn(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 2); }
template <typename T, int B>
__device__ inline int slot_turn(int line) {
  return (sizeof(T) == 2 ? (line & 1) << 2 | (line & 2) | (line >> 3 & 1) : line >> 2 & 3) & (B / 16 - 1);
}
template <typename T>
__device__ inline int part_turn(int line) {
  return sizeof(T) == 2 ? line >> 1 & 1 : line >> 2 & 3;
}

// Which row of R, in the wave's part, is row q of its fragment j, and so which
// columns of C lane group g (of 16 lanes) holds: with Runs eight neighbouring
// ones in two fragments, which 16-bit results are stored by (16 bytes a lane,
// 64 a row); else four of every 16, for single-precision ones.
template <bool Runs>
struct Order {
  static __device__ int row(int j, int q) {
    return Runs ? (j >> 1) * 32 + (q >> 2) * 8 + (j & 1) * 4 + (q & 3) : j * 16 + q;
  }
  static __device__ int col(int j, int g) { return Runs ? (j >> 1) * 32 + g * 8 + (j & 1) * 4 : j * 16 + g * 4; }
};

template <typename T, int B, int WAVES, typename Op>
struct Stage {
  static constexpr int LOADS = B / 16 / WAVES;
  static_assert(LOADS >= 1 && B % (16 * WAVES) == 0, "every wave loads the same number of times");
  static constexpr int LINE = B * int(sizeof(T));  // bytes, rows contiguous
  // rows contiguous: lines from one load of a wave to its next
  static constexpr int NEXT = Op::kContiguous ? 0 : WAVES * 1024 / LINE;
  static_assert(Op::kContiguous || (WAVES * 1024) % LINE == 0, "a wave's loads are whole lines apart");
  static constexpr int WAVES_ = WAVES, ROWS = B;
  static constexpr bool CONTIGUOUS = Op::kContiguous;
  const char *src[LOADS];
  int k0;  // of the lane's chunk in a step, in the first load

  __device__ void aim(const Op &op, int row0, int wave, int lane) {
    if (Op::kContiguous) {
      k0 = ((lane & 3) ^ chunk_turn(wave * 16 + (lane >> 2))) * kChunk<T>;  // the same in every load
#pragma unroll
      for (int i = 0; i < LOADS; ++i) src[i] = op.base(row0 + (i * WAVES + wave) * 16 + (lane >> 2), k0);
    } else {
      k0 = (wave * 1024 + lane * 16) / LINE;
      const int part = (wave * 1024 + lane * 16) % LINE / 16;
      constexpr int per_slot = int(sizeof(T));  // 16-byte parts of 16 elements
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int line = k0 + i * NEXT, slot = (part / per_slot) ^ slot_turn<T, B>(line);
        src[i] = op.base(row0 + slot * 16 + ((part % per_slot) ^ part_turn<T>(line)) * kChunk<T>, line);
      }
    }
  }
  // where a lane's load i of a step comes from
  __device__ const char *from(const Op &op, int step, int64_t ahead, int i) const {
    return op.in(step, k0 + i * NEXT) ? src[i] + ahead : reinterpret_cast<const char *>(&kZeroChunk);
  }
};

// 1 KiB into LDS at `to` (the same for all lanes), 16 bytes from each lane's
// `from`.  In assembly, since the compiler waits for every load into LDS that it
// knows to be in flight before it reads LDS, whichever stage either is of: here
// stage_barrier waits, and the clobbered memory keeps reads on their side of it.
// No register is written; `s_nop` is the state between M0 and its use.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // M0 in the clobbers: reserved, so the compiler sets it where it uses it
__device__ inline void load_to_lds(const char *from, lds_char *to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(uint32_t(uintptr_t(to))), "v"(from)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// The loads of an operand's part of a step into its stage.
template <typename S, typename Op>
__device__ inline void load_step(const S &stage, const Op &op, int step, int wave, lds_char *to) {
  const int64_t ahead = op.ahead(step);
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) load_to_lds(stage.from(op, step, ahead, i), to + (i * S::WAVES_ + wave) * 1024);
}

// A wave's fragments of a step, from row `row0` of the operand's part on.
template <typename T, typename S, typename Order, int N>
__device__ inline void read_fragments(u32x4 (&f)[N], const lds_char *tile, int row0, int lane) {
  const int q = lane & 15, group = lane >> 4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (S::CONTIGUOUS) {
      const int row = row0 + Order::row(i, q);
      f[i] = *(const lds_u32x4 *)(tile + row * 64 + (group ^ chunk_turn(row)) * 16);
    } else if constexpr (sizeof(T) == 2) {
      // lane q reads four rows of line q / 4: those that lanes 4 (q % 4) on get
      const int line = group * 8 + (q >> 2), row = row0 + Order::row(i, (q & 3) * 4);
      const int at = line * S::LINE + ((row >> 4) ^ slot_turn<T, S::ROWS>(line)) * 32 +
                     (((row & 15) * 2) ^ (part_turn<T>(line) * 16));
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at)));
      const u32x2 hi =
          __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + at + 4 * S::LINE)));
      f[i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int line = group * 4 + e, row = row0 + Order::row(i, q);
        f[i][e] = *(const lds_u32 *)(tile + line * S::LINE + ((row >> 4) ^ slot_turn<T, S::ROWS>(line)) * 64 +
                                     (((row >> 2 & 3) ^ part_turn<T>(line)) * 16 + (row & 3) * 4));
      }
    }
  }
}

// Every wave's reads and its older loads are done; those of the last `Flying`
// loads of each wave may be in flight.
template <int Flying>
__device__ inline void stage_barrier() {
  static_assert(Flying < 16, "vmcnt's low field");
  __builtin_amdgcn_s_waitcnt(0x0070 | Flying);  // vmcnt(Flying) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// C tiles of BM x BN by WM x WN waves, on a grid that stays on the device and
// walks through the tiles.  Four stages in LDS: while a step's fragments are
// multiplied, the next step's are read and three steps' loads are in flight.
// The loads run over the ends of tiles, so that a tile's first steps are there
// when the epilogue of the tile before is done.
// Between two barriers the stage that is filled is not the one that is read.
//
// What bounds it: a CU takes 64 bytes a cycle from its L2, so that at the
// matrix unit's rate a 128 x 128 tile needs all of that and a 256 x 256 tile
// half; 256 x 256 with one step in flight was bound by the loads' latency.  Now
// (8192 x 1024 x 16384 of bf16, two splits, 229 to 242 us = 1,140 to 1,200
// TFLOP/s, where a library product of 8192^3 reaches 1,323) the matrix unit is
// busy 59% of the cycles, at a clock of about 1.8 GHz (2.4 GHz at most).
template <typename T, int BM, int BN, int WM, int WN, typename L, typename R, typename Epilogue>
__device__ inline void walk_tiles(const Grid &g, const L &left, const R &right, const Epilogue &epilogue,
                                  lds_char *stages, char *scratch) {
  constexpr int TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16, WAVES = WM * WN;
  constexpr int STAGE = (BM + BN) * 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  typedef Stage<T, BM, WAVES, L> StageL;
  typedef Stage<T, BN, WAVES, R> StageR;
  constexpr int LOADS = StageL::LOADS + StageR::LOADS;
  typedef Order<false> OrderL;
  typedef Order<Epilogue::kRuns> OrderR;

  // this workgroup's items (a tile and a split of k): every width-th of its
  // die's run of them
  const int tiles = g.mtiles * g.ntiles, items = tiles * g.splits;
  const int per = (items + 7) >> 3, width = int(gridDim.x >> 3);
  const int last = min(items, (int(blockIdx.x & 7) + 1) * per);
  int item = int(blockIdx.x & 7) * per + int(blockIdx.x >> 3);
  if (item >= last) return;

  // the loads' place in the items; at their end the last step is loaded once
  // more, so that every wave has the same number of loads in flight
  StageL from_l;
  StageR from_r;
  int ahead_item = item, ahead_step, ahead_end;
  auto aim = [&]() {
    int mt, nt;
    tile_at(g, ahead_item % tiles, mt, nt);
    ahead_step = ahead_item / tiles * g.split;
    ahead_end = min(g.steps, ahead_step + g.split);
    from_l.aim(left, mt * BM, wave, lane);
    from_r.aim(right, nt * BN, wave, lane);
  };
  auto advance = [&]() {
    if (ahead_step + 1 < ahead_end) {
      ++ahead_step;
    } else if (ahead_item + width < last) {
      ahead_item += width;
      aim();
    }
  };
  f32x4 acc[MI][NI];
  // an instruction never follows one with the same accumulators
  auto multiply = [&](const u32x4(&l)[MI], const u32x4(&r)[NI]) {
#pragma unroll
    for (int e = 0; e < (sizeof(T) == 4 ? 4 : 1); ++e)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          if constexpr (sizeof(T) == 4) acc[i][j] = mma_one(r[j], l[i], e, acc[i][j]);
          else acc[i][j] = mma<T>(r[j], l[i], acc[i][j]);
        }
  };

  auto load = [&](int stage) {
    load_step(from_l, left, ahead_step, wave, stages + stage * STAGE);
    load_step(from_r, right, ahead_step, wave, stages + stage * STAGE + BM * 64);
  };
  auto read = [&](int stage, u32x4(&l)[MI], u32x4(&r)[NI]) {
    read_fragments<T, StageL, OrderL>(l, stages + stage * STAGE, wm * TM, lane);
    read_fragments<T, StageR, OrderR>(r, stages + stage * STAGE + BM * 64, wn * TN, lane);
  };
  // the loads' addresses of two transposed operands do not fit beside the
  // fragments that are read
  constexpr bool kLoadsFirst = !L::kContiguous && !R::kContiguous;
  auto read_or_load = [&](int from, u32x4(&l)[MI], u32x4(&r)[NI], int to) {
    if constexpr (kLoadsFirst) load(to);
    read(from, l, r);
    if constexpr (!kLoadsFirst) load(to);
  };

  aim();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    load(i);
    advance();
  }
  stage_barrier<0>();
  u32x4 al[MI], ar[NI], bl[MI], br[NI];
  read(0, al, ar);
  int slot = 0;  // the stage of the step that is multiplied
  for (; item < last; item += width) {
    int mt, nt;
    tile_at(g, item % tiles, mt, nt);
    const int split = item / tiles;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
    // a step: the next one's fragments are read (past the last step: the last
    // one's once more, which nothing uses), and its own stage, which every wave
    // has read, is loaded
    for (int steps = min(g.split, g.steps - split * g.split); steps > 0; steps -= 2) {
      stage_barrier<2 * LOADS>();
      const int odd = (slot + 1) & 3, even = (slot + 2) & 3;
      read_or_load(odd, bl, br, slot);
      multiply(al, ar);
      advance();
      stage_barrier<2 * LOADS>();
      read_or_load(even, al, ar, odd);
      multiply(bl, br);
      advance();
      slot = even;
    }
    epilogue(Place{mt * BM + wm * TM, nt * BN + wn * TN, mt, nt, wm, wn, lane, split, scratch}, acc);
  }
}

// BM x BN = 256 x 256: eight waves of 128 x 64, one workgroup a CU.  128 x 128
// and 64 x 64, where those leave CUs without work: four waves, several
// workgroups a CU.
template <typename T, int BM, int BN, int WM, int WN, typename L, typename R, typename Epilogue>
__global__ __launch_bounds__(64 * WM *WN, 2) void k_product(Grid g, L left, R right, Epilogue epilogue) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  walk_tiles<T, BM, BN, WM, WN>(g, left, right, epilogue, (lds_char *)lds, lds + 4 * (BM + BN) * 64);
}

// ------------------------------------------------------------- epilogues ----
// At the head of an epilogue's row of fragments: no work of other rows is mixed
// with this one's (beside 128 accumulators there are no registers for it).
__device__ inline void one_row_at_a_time() { __builtin_amdgcn_sched_barrier(0); }

// Four columns of a row, of which `count` are inside it, at any address (global
// memory takes vectors wherever they begin; element by element the gradient of
// 111968 x 318 of f16 from 123 rows took 96 us instead of 41).
template <typename T>
__device__ inline void store4(T *p, f32x4 v, int count) {
  if (count >= 4) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    *reinterpret_cast<vec *>(p) = vec{T(v[0]), T(v[1]), T(v[2]), T(v[3])};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < count) p[r] = T(v[r]);
  }
}

template <typename T>
__device__ inline f32x4 load4(const T *p, int count) {
  f32x4 v = {0, 0, 0, 0};
  if (count >= 4) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
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

// Stores the columns of C that a lane of group g holds, in a row that ends at
// `cols`: with Runs and 16-bit types eight at a time.
template <bool Runs, typename T, int NI, typename Value>
__device__ inline void store_row(T *row, int n0, int g, int cols, Value value) {
#pragma unroll
  for (int j = 0; j < NI; j += 2) {
    const int c = n0 + Order<Runs>::col(j, g), d = n0 + Order<Runs>::col(j + 1, g);
    const f32x4 a = value(j), b = value(j + 1);
    if (Runs && sizeof(T) == 2 && c + 8 <= cols) {
      typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
      *reinterpret_cast<vec *>(row + c) = vec{T(a[0]), T(a[1]), T(a[2]), T(a[3]), T(b[0]), T(b[1]), T(b[2]), T(b[3])};
    } else {
      if (c < cols) store4(row + c, a, cols - c);
      if (d < cols) store4(row + d, b, cols - d);
    }
  }
}

// Where row m of a product's result goes: a matrix, or w_gate's and w_value's
// gradients in turns of four rows (pair_row).
template <typename T>
struct Target {
  T *p, *q;
  int64_t ld;
  int rows;  // of p (and q)
  bool pair;
  const float *factor;  // of the result, on the device: one for all (step 0) or one a row (step 1); NULL = 1
  int factor_step;
  __device__ float scale(int m) const { return factor ? factor[m * factor_step] : 1.0f; }
  __device__ T *row(int m) const {
    const int f = pair ? pair_row(m) : m;
    if (f >= rows) return nullptr;
    return (pair && (m & 4) ? q : p) + f * ld;
  }
};

template <typename T>
struct Store {
  static constexpr bool kRuns = sizeof(T) == 2;
  Target<T> out;
  int cols;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      const int m = at.m0 + i * 16 + (at.lane & 15);
      T *row = out.row(m);
      if (!row) continue;
      const float f = out.scale(m);
      store_row<kRuns, T, NI>(row, at.n0, at.lane >> 4, cols, [&](int j) { return c[i][j] * f; });
    }
  }
};

// One split's part of the result, in 32 bits: [split][rows][cols4], added to
// what an earlier launch left there if Add.
template <bool Add>
struct StorePart {
  static constexpr bool kRuns = false;
  float *part;
  int rows, cols4;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
      float *row = part + (int64_t(at.split) * rows + m) * cols4;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = at.n0 + Order<kRuns>::col(j, at.lane >> 4);
        if (n >= cols4) continue;
        f32x4 *p = reinterpret_cast<f32x4 *>(row + n);
        if constexpr (Add) *p += c[i][j];
        else *p = c[i][j];
      }
    }
  }
};

// In half precision operands of gradients are brought into the type's range, by
// powers of two from the sizes of the rows that they are made of.
template <typename T>
constexpr bool kScaledRows = false;
template <>
constexpr bool kScaledRows<f16> = true;

// The activation and its derivative, for matrices of type T.  In 16-bit types the
// normal distribution function by Abramowitz and Stegun, 7.1.26:
// 1 - Phi(|a|) = exp(-a^2 / 2) (a1 t + .. + a5 t^5) / 2 with t = 1 / (1 + p |a| / sqrt 2),
// within 7.5e-8 (not of itself: of 1), and the exponential is the derivative's
// too.  In single precision that is more than Phi's rounding where it is small:
// the complementary error function.
template <typename T>
__device__ inline void gate(int act, float a, float &p, float &dp) {
  if constexpr (sizeof(T) == 4) {
    if (act == LDA_GELU) {
      const float phi = 0.5f * erfcf(-0.70710678118654752f * a);
      p = a * phi;
      dp = phi + a * 0.3989422804014327f * expf(-0.5f * a * a);
      return;
    }
  } else if (act == LDA_GELU) {
    const float bell = __builtin_amdgcn_exp2f(-0.5f * kLog2e * a * a);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * 0.70710678118654752f * fabsf(a));
    const float tail = 0.5f * bell * t *
                       (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float phi = a >= 0.0f ? 1.0f - tail : tail;
    p = a * phi;
    dp = phi + a * 0.3989422804014327f * bell;
    return;
  }
  // sigmoid(a) and 1 - sigmoid(a) from e = exp(-|a|), which does not overflow
  const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(a)), big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  const float s = a >= 0.0f ? big : small, t = a >= 0.0f ? small : big;
  if (act == LDA_SIGMOID) {
    p = s;
    dp = s * t;
  } else {
    p = a * s;
    dp = s + a * s * t;
  }
}

// h from the accumulators: a and b are never written.  8192 x 1024 x 4096 of
// bf16: 149 to 157 us = 875 to 920 TFLOP/s of both projections, the activation
// included.
template <typename T>
struct GatedForward {
  static constexpr bool kRuns = true;
  T *h;
  int64_t ld;
  int rows, hidden, act;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
#pragma unroll
      for (int j = 0; j < NI; j += 2) {  // a and b of the same four columns
        const int f = pair_row(at.n0 + Order<kRuns>::col(j, at.lane >> 4));
        if (f >= hidden) continue;
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p, dp;
          gate<T>(act, c[i][j][r], p, dp);
          v[r] = p * c[i][j + 1][r];
        }
        store4(h + m * ld + f, v, hidden - f);
      }
    }
  }
};

// da and db in turns of four columns (pair_row), zero past `hidden`: operands of
// the backward products, from a and b recomputed.  Kept in 32 bits, as their
// precision asks for, they would be written and read again (268 MB each way at
// 8192 x 4096, about 110 us); recomputed, they cost 150 us of the backward
// pass' 500, and a training step keeps x alone.  192 us with dh's reads and
// dab's stores.
//
// In half precision da and db go past the type's range, or below it, long before
// the gradients that are made of them: each row is multiplied by a power of two
// (k_gated_scales), which the products' results or operands take back.
template <typename T>
struct GatedBackward {
  static constexpr bool kRuns = true;
  const T *dh;
  int64_t ld;
  const float *scale;  // of each row, with kScaledRows
  T *dab;              // [rows][pair_cols]
  int rows, hidden, pair_cols, act;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      const int m = at.m0 + i * 16 + (at.lane & 15);
      if (m >= rows) continue;
      float s = 1.0f;
      if constexpr (kScaledRows<T>) s = scale[m];
      f32x4 d[NI];
#pragma unroll
      for (int j = 0; j < NI; j += 2) {
        const int f = pair_row(at.n0 + Order<kRuns>::col(j, at.lane >> 4));
        f32x4 dhv = load4(dh + m * ld + f, hidden - f);
        if constexpr (kScaledRows<T>) dhv *= s;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float p, dp;
          gate<T>(act, c[i][j][r], p, dp);
          d[j][r] = f + r < hidden ? dhv[r] * c[i][j + 1][r] * dp : 0.0f;
          d[j + 1][r] = f + r < hidden ? dhv[r] * p : 0.0f;
        }
      }
      store_row<kRuns, T, NI>(dab + int64_t(m) * pair_cols, at.n0, at.lane >> 4, pair_cols, [&](int j) { return d[j]; });
    }
  }
};

__device__ inline float exp_diff(float z, float top) { return __builtin_amdgcn_exp2f((z - top) * kLog2e); }

// Two parts of a softmax: (largest logit, sum of exp(z - it)).
__device__ inline float2 softmax_join(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.0f : top;
  return make_float2(top, a.y * exp_diff(a.x, ref) + b.y * exp_diff(b.x, ref));
}

// The bias of a lane's words; -inf past the vocabulary, where the products are
// of some row of the weights that is in it.
template <bool Runs, int NI>
__device__ inline void word_bias(f32x4 (&b)[NI], const float *bias, int n0, int lane, int first, int vocab) {
#pragma unroll
  for (int j = 0; j < NI; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int v = first + n0 + Order<Runs>::col(j, lane >> 4) + r;
      b[j][r] = bias ? bias[min(v, vocab - 1)] : 0.0f;
      if (v >= vocab) b[j][r] = -INFINITY;
    }
}

// Where a row's label is among the wave's words, if this lane holds it: 4 j + r,
// else -1.
template <bool Runs, int NI>
__device__ inline int label_at(int label, int n0, int lane, int first, int vocab) {
  const int at = label - first - n0;
  if (label < 0 || label >= vocab || at < 0 || at >= NI * 16) return -1;
  if (Runs) return (at >> 3 & 3) == lane >> 4 ? (at >> 5) * 8 + (at & 7) : -1;
  return (at >> 2 & 3) == lane >> 4 ? (at >> 4) * 4 + (at & 3) : -1;
}

// Per row and tile of words: the largest logit and the sum of exp(z - it), and
// the label's logit from the lane that holds it.  The parts of a row, one of a
// tile's 256 words each, are joined by k_lse_join: 36 MB for 8,192 rows and
// 141,000 words, where the logits would be 2.3 GB.
//
// 8192 x 1024 x 141000 of bf16: 2.1 to 2.25 ms = 1,050 to 1,120 TFLOP/s with
// this epilogue (a library product that writes the logits: 1,044).  A wave's
// exponentials do not overlap with its own products.
//
// With a Teacher the logits are multiplied by `unit` (1 / temperature) and there
// is no label.
template <int BM, int WN, bool Teacher = false>
struct SoftmaxPart {
  static constexpr bool kRuns = false;
  const float *bias;
  const int32_t *labels;
  float *label_logit;  // [rows]
  float2 *part;        // [ntiles][rows]
  int rows, vocab;
  float unit;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
    float2 *shared = reinterpret_cast<float2 *>(at.lds);  // [WN][BM]
    f32x4 b[NI];
    word_bias<kRuns>(b, bias, at.n0, at.lane, 0, vocab);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      f32x4 z[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        z[j] = c[i][j] + b[j];
        if constexpr (Teacher) z[j] *= unit;
      }
      if constexpr (!Teacher) {
        const int m = at.m0 + i * 16 + (at.lane & 15);
        const int hit = label_at<kRuns, NI>(m < rows ? labels[m] : -1, at.n0, at.lane, 0, vocab);
        if (__ballot(hit >= 0)) {
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (hit == j * 4 + r) label_logit[m] = z[j][r];
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, z[j][r]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      // nothing but -inf: the sum is 0 against any finite reference
      const float ref = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += exp_diff(z[j][r], ref);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (at.lane < 16) shared[at.wn * BM + at.wm * MI * 16 + i * 16 + at.lane] = make_float2(top, sum);
    }
    __syncthreads();
    const int m = at.mt * BM + int(threadIdx.x);
    if (threadIdx.x < BM && m < rows) {
      float2 a = shared[threadIdx.x];
#pragma unroll
      for (int w = 1; w < WN; ++w) a = softmax_join(a, shared[w * BM + threadIdx.x]);
      part[int64_t(at.nt) * rows + m] = a;
    }
  }
};

// G of one piece of the vocabulary (words from `first` on) without the rows'
// own gradients, S (exp(z - lse) - [v = label]), and the column sums of the
// rows' gradients times it by tile of rows.  Where one value of G leads its row
// it is the label's, -S (1 - p), which rounds to -S itself where p is small; so
// what the rounding of G to bf16 or f16, as operand of two products, changes is
// small beside it.  S is 1, in half precision 2^14, so that probabilities down
// to 2^-28 are normal numbers.
//
// A piece of 16,384 words at 8,192 rows of width 1,024: 301 to 317 us, where dx,
// a product of the same size that stores little, takes 229 to 242: the rest is
// the exponentials and G's 268 MB.
template <typename T>
constexpr float kGradLog2 = 0.0f;
template <>
constexpr float kGradLog2<f16> = 14.0f;
template <typename T>
constexpr float kGradUnit = 1.0f;
template <>
constexpr float kGradUnit<f16> = 16384.0f;

//
// With a Teacher the logits are multiplied by `unit`, `labels` says only which
// rows are kept (0) or left out (-1), and G lacks what the teacher gives its
// words, which k_teacher_words puts right; `rest` (NULL: not wanted) gets what the
// rounding of G left.
template <typename T, int BN, int WM, bool Teacher = false>
struct SoftmaxGrad {
  static constexpr bool kRuns = true;
  const float *bias;
  const int32_t *labels;
  const float *lse, *row_factor;  // row_factor: dloss / S, 0 for a row that is left out
  T *grad;                        // [rows][ldg]
  int64_t ldg;
  float *col_part;  // [mtiles][piece], NULL without a bias
  int rows, vocab, first, piece;
  float unit;
  T *rest;
  template <int MI, int NI>
  __device__ void operator()(const Place &at, f32x4 (&c)[MI][NI]) const {
    f32x4 b[NI], sums[NI];
    word_bias<kRuns>(b, bias, at.n0, at.lane, first, vocab);
#pragma unroll
    for (int j = 0; j < NI; ++j) sums[j] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      one_row_at_a_time();
      const int m = at.m0 + i * 16 + (at.lane & 15);
      const int label = m < rows ? labels[m] : -1;
      const float l = m < rows ? lse[m] : 0.0f, d = m < rows ? row_factor[m] : 0.0f;
      const bool kept = label >= 0 && label < vocab && l != -INFINITY;
      f32x4 z[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float logit = c[i][j][r] + b[j][r];
          if constexpr (Teacher) logit *= unit;
          z[j][r] = kept ? __builtin_amdgcn_exp2f((logit - l) * kLog2e + kGradLog2<T>) : 0.0f;
        }
      if constexpr (!Teacher) {
        const int hit = kept ? label_at<kRuns, NI>(label, at.n0, at.lane, first, vocab) : -1;
        if (__ballot(hit >= 0)) {
#pragma unroll
          for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (hit == j * 4 + r) z[j][r] -= kGradUnit<T>;
        }
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) sums[j] += z[j] * d;
      if (m < rows)
        store_row<kRuns, T, NI>(grad + m * ldg, at.n0, at.lane >> 4, int(ldg), [&](int j) { return z[j]; });
      if constexpr (Teacher && sizeof(T) == 2 && BN < 256) {  // few rows have smaller tiles
        if (rest && m < rows)
          store_row<kRuns, T, NI>(rest + m * ldg, at.n0, at.lane >> 4, int(ldg), [&](int j) {
            f32x4 left;
#pragma unroll
            for (int r = 0; r < 4; ++r) left[r] = z[j][r] - float(T(z[j][r]));
            return left;
          });
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
        if ((at.lane & 15) == 0) shared[at.wm * BN + at.wn * NI * 16 + Order<kRuns>::col(j, at.lane >> 4) + r] = s;
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
};

// ---------------------------------------------------------------- few rows ---
// At most 16 rows of x (single tokens in serving): the weights are read once,
// from HBM straight into fragments, 16 of their rows a wave, and nothing is
// staged; x comes from the caches.  Bound by the weights' bytes: one row against
// 141000 x 1024 of bf16 (289 MB) takes 55 us = 5.3 TB/s, where a copy of 4 GiB
// reaches 4.8 TB/s; through tiles of 64 x 64 it took 83 us.
constexpr int kFewRows = 16;

// Chunk `c` of a row of `cols` elements, zero past its end; a chunk that a row
// ends inside of element by element.
template <typename T, bool Aligned>
__device__ inline u32x4 row_chunk(const T *row, int c, int cols) {
  if (Aligned) return c * kChunk<T> < cols ? *reinterpret_cast<const u32x4 *>(row + c * kChunk<T>) : u32x4{0, 0, 0, 0};
  typedef T vec __attribute__((ext_vector_type(kChunk<T>), aligned(sizeof(T))));
  vec v;
  if ((c + 1) * kChunk<T> <= cols) {
    v = *reinterpret_cast<const vec *>(row + c * kChunk<T>);
  } else {
#pragma unroll
    for (int e = 0; e < kChunk<T>; ++e) v[e] = c * kChunk<T> + e < cols ? row[c * kChunk<T> + e] : T(0.0f);
  }
  return __builtin_bit_cast(u32x4, v);
}

// Products of TILES x 16 rows of weights (this lane's: w[t]) with x, over the
// groups of four chunks part, part + parts, ..: C[m = lane & 15][n = 4 (lane >> 4) + r].
template <typename T, bool Aligned, int TILES>
__device__ inline void few_products(const T *x, const T *const (&w)[TILES], int cols, int part, int parts, int lane,
                                    f32x4 (&c)[TILES]) {
  constexpr int U = 8 / TILES;  // groups in flight
  const int groups = (cols + 4 * kChunk<T> - 1) / (4 * kChunk<T>);
#pragma unroll
  for (int t = 0; t < TILES; ++t) c[t] = f32x4{0, 0, 0, 0};
  for (int g = part; g < groups; g += parts * U) {
    u32x4 xv[U], wv[U][TILES];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int chunk = (g + u * parts) * 4 + (lane >> 4);
#pragma unroll
      for (int t = 0; t < TILES; ++t) wv[u][t] = row_chunk<T, Aligned>(w[t], chunk, cols);
      xv[u] = row_chunk<T, Aligned>(x, chunk, cols);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < TILES; ++t) c[t] = mma<T>(wv[u][t], xv[u], c[t]);
  }
}

// 16 columns of h a workgroup; its four waves share the sum over k (a hidden
// width of 1,024 is 64 workgroups: 5 us at a width of 1,000, latency).
template <typename T, bool Aligned>
__global__ __launch_bounds__(256) void k_gated_few(const T *x, int64_t ldx, const T *gates, int64_t ld_gate,
                                                   const T *values, int64_t ld_value, int rows, int width, int hidden,
                                                   int act, T *h, int64_t ldh) {
  __shared__ f32x4 shared[3][2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15;
  const int64_t n = min(int(blockIdx.x) * 16 + q, hidden - 1);
  const T *const w[2] = {gates + n * ld_gate, values + n * ld_value};
  f32x4 c[2];
  few_products<T, Aligned, 2>(x + min(q, rows - 1) * ldx, w, width, wave, 4, lane, c);
  if (wave) {
    shared[wave - 1][0][lane] = c[0];
    shared[wave - 1][1][lane] = c[1];
  }
  __syncthreads();
  if (wave || q >= rows) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    c[0] += shared[i][0][lane];
    c[1] += shared[i][1][lane];
  }
  const int f = int(blockIdx.x) * 16 + (lane >> 4) * 4;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    float p, dp;
    gate<T>(act, c[0][r], p, dp);
    if (f + r < hidden) h[q * ldh + f + r] = T(p * c[1][r]);
  }
}

// Each wave takes every (4 gridDim.x)-th 16 words and keeps its lanes' softmax
// so far; part [rows][gridDim.x].  With a Teacher as SoftmaxPart.
template <typename T, bool Aligned, bool Teacher>
__global__ __launch_bounds__(256) void k_xent_few(const T *x, int64_t ldx, const T *weight, int64_t ldw,
                                                  const float *bias, const int32_t *labels, int rows, int width,
                                                  int vocab, float unit, float *label_logit, float2 *part) {
  __shared__ float2 shared[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15;
  const T *row = x + min(q, rows - 1) * ldx;
  int label = -1;
  if constexpr (!Teacher) label = q < rows ? labels[q] : -1;
  float2 so_far = make_float2(-INFINITY, 0.0f);
  for (int n0 = (int(blockIdx.x) * 4 + wave) * 16; n0 < vocab; n0 += int(gridDim.x) * 64) {
    const T *const w[1] = {weight + int64_t(min(n0 + q, vocab - 1)) * ldw};
    f32x4 c[1];
    few_products<T, Aligned, 1>(row, w, width, 0, 1, lane, c);
    const int v = n0 + (lane >> 4) * 4;
    float top = so_far.x;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      c[0][r] = v + r < vocab ? (bias ? c[0][r] + bias[v + r] : c[0][r]) : -INFINITY;
      if constexpr (Teacher) c[0][r] *= unit;
      else if (v + r == label && label < vocab) label_logit[q] = c[0][r];
      top = fmaxf(top, c[0][r]);
    }
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = so_far.y * exp_diff(so_far.x, ref);
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += exp_diff(c[0][r], ref);
    so_far = make_float2(top, sum);
  }
#pragma unroll
  for (int x_ = 16; x_ < 64; x_ <<= 1)
    so_far = softmax_join(so_far, make_float2(__shfl_xor(so_far.x, x_), __shfl_xor(so_far.y, x_)));
  if (lane < 16) shared[wave][lane] = so_far;
  __syncthreads();
  if (threadIdx.x >= rows) return;
  for (int i = 1; i < 4; ++i) so_far = softmax_join(so_far, shared[i][threadIdx.x]);
  part[int64_t(threadIdx.x) * gridDim.x + blockIdx.x] = so_far;
}

// ---------------------------------------------------------- small kernels ---
// The loss of a row from its softmax (largest logit, sum); without labels only
// the logarithm.
__device__ inline void write_loss(float2 a, int m, const float *label_logit, const int32_t *labels, int vocab,
                                  float *loss, float *lse) {
  const float total = a.x == -INFINITY && a.y == 0.0f ? -INFINITY : a.x + kLn2 * __builtin_amdgcn_logf(a.y);
  lse[m] = total;
  if (!labels) return;
  const int label = labels[m];
  float out = 0.0f;
  if (label >= 0 && label < vocab) {
    const float z = label_logit[m];
    out = z == -INFINITY ? INFINITY : total - z;
  }
  loss[m] = out;
}

// Joins the parts [ntiles][rows]: 16 rows a workgroup, 16 threads a row.
__global__ __launch_bounds__(256) void k_lse_join(const float2 *part, int ntiles, const float *label_logit,
                                                  const int32_t *labels, int rows, int vocab, float *loss, float *lse) {
  __shared__ float2 shared[16][17];
  const int m = blockIdx.x * 16 + (threadIdx.x & 15), way = threadIdx.x >> 4;
  float2 a = make_float2(-INFINITY, 0.0f);
  if (m < rows)
#pragma unroll 8
    for (int t = way; t < ntiles; t += 16) a = softmax_join(a, part[int64_t(t) * rows + m]);
  shared[way][threadIdx.x & 15] = a;
  __syncthreads();
  if (threadIdx.x < 16 && m < rows) {
    for (int w = 1; w < 16; ++w) a = softmax_join(a, shared[w][threadIdx.x]);
    write_loss(a, m, label_logit, labels, vocab, loss, lse);
  }
}

// Joins the parts [rows][parts] of few rows: one workgroup a row.
__global__ __launch_bounds__(256) void k_lse_join_few(const float2 *part, int parts, const float *label_logit,
                                                      const int32_t *labels, int vocab, float *loss, float *lse) {
  __shared__ float2 shared[4];
  const int m = blockIdx.x;
  float2 a = make_float2(-INFINITY, 0.0f);
  for (int t = threadIdx.x; t < parts; t += 256) a = softmax_join(a, part[int64_t(m) * parts + t]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) a = softmax_join(a, make_float2(__shfl_xor(a.x, x), __shfl_xor(a.y, x)));
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = a;
  __syncthreads();
  if (threadIdx.x) return;
  for (int w = 1; w < 4; ++w) a = softmax_join(a, shared[w]);
  write_loss(a, m, label_logit, labels, vocab, loss, lse);
}

// The largest of the threads' values, for every thread of 1,024.
__device__ inline float group_max(float v, float (&shared)[16]) {
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) v = fmaxf(v, __shfl_xor(v, x));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) v = fmaxf(v, shared[w]);
  return v;
}

// The rows' gradients as factors of the products: row_factor = dloss / S for dx
// and dbias, and x_factor = dloss / unit for the rows of x in dweight, whose
// result is then multiplied by out[0] = unit / S.  The unit is the smallest
// finite |dloss| above 0, by the power of two that brings it to the largest or
// just above: equal gradients, and power-of-two multiples of one (a word that
// counts once, twice, four times), then leave the rows of x unrounded, and no
// factor is above 1, so that none takes x out of its type's range.  The factors
// are 0 for rows that are left out.
//
// In half precision (x_size: the rows' sizes) another power of two brings
// the largest |x| |dloss| to 2^14 or above, below 2^15: rows lose bits only where
// theirs is more than some 2^28 below, instead of where |dloss| is 2^10 to 2^14
// below the largest.
__global__ __launch_bounds__(1024) void k_grad_factors(const float *dloss, const float *lse, const int32_t *labels,
                                                       const float2 *x_size, int rows, int vocab, float s, float *out,
                                                       float *row_factor, float *x_factor) {
  __shared__ float shared[16];
  auto in = [&](int m) { return labels[m] >= 0 && labels[m] < vocab; };
  float top = 0.0f, low = INFINITY;
  for (int m = threadIdx.x; m < rows; m += 1024) {
    const float d = fabsf(dloss[m]);
    if (in(m) && d < INFINITY && d > 0.0f) {
      top = fmaxf(top, d);
      low = fminf(low, d);
    }
  }
  top = group_max(top, shared);
  low = -group_max(-low, shared);
  float unit = x_size ? 0x1p-70f : 0x1p-100f;  // at least: below, the quotients would leave the range
  if (top > unit) {
    int e_top, e_low;
    frexpf(top, &e_top);
    unit = ldexpf(frexpf(low, &e_low), e_top);
    if (unit < top) unit = fminf(2.0f * unit, 0x1.fffffep127f);
  }
  float shift = 1.0f;
  if (x_size) {
    float most = 0.0f;
    for (int m = threadIdx.x; m < rows; m += 1024) {
      const float d = fabsf(dloss[m]);
      if (in(m) && lse[m] != -INFINITY && d < INFINITY) most = fmaxf(most, x_size[m].x * (d / unit));
    }
    most = group_max(most, shared);
    int e = 15;
    if (most > 0.0f) frexpf(most, &e);  // most < 2^e
    shift = ldexpf(1.0f, 15 - (e < -25 ? -25 : e));
  }
  if (threadIdx.x == 0) out[0] = unit / s / shift;
  for (int m = threadIdx.x; m < rows; m += 1024) {
    const bool kept = in(m) && lse[m] != -INFINITY;
    row_factor[m] = kept ? dloss[m] / s : 0.0f;
    x_factor[m] = kept ? dloss[m] / unit * shift : 0.0f;
  }
}

// out[n] = sum over t of part[t][n], less what `less` has there (NULL = 0): 64
// columns a workgroup, a wave for every fourth part.
__global__ __launch_bounds__(256) void k_sum_parts(const float *part, int count, int n_all, const float *less,
                                                   float *out) {
  __shared__ float shared[4][64];
  const int n = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  float s = 0.0f;
  if (n < n_all) {
#pragma unroll 4
    for (int t = wave; t < count; t += 4) s += part[int64_t(t) * n_all + n];
  }
  shared[wave][threadIdx.x & 63] = s;
  __syncthreads();
  if (wave == 0 && n < n_all) {
    s = s + shared[1][threadIdx.x] + shared[2][threadIdx.x] + shared[3][threadIdx.x];
    out[n] = less ? s - less[n] : s;
  }
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
#pragma unroll 8
    for (int z = 1; z < splits; ++z) s += *reinterpret_cast<const f32x4 *>(part + z * all + at);
    s *= out.scale(m);
    store4(row + n, s, cols - n);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero(T *p, int64_t n) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = T(0.0f);
}

// Copies of matrices for the products, up to four a launch (a launch takes
// longer than the copy of a small matrix): rows at multiples of 16 bytes, zero
// past their end; each row times its factor, a row of factor 0 zero whatever it
// holds (factor NULL = 1).  A lane reads a chunk at once, from wherever it begins,
// and the one that the row ends in element by element; divisions in 32 bits where
// the count of chunks allows it.
template <typename T>
struct Copy {
  const T *src;
  int64_t ld, rows;
  int cols, chunks;  // of a row of dst
  const float *factor;
  T *dst;
};
constexpr int kCopies = 4;
template <typename T>
struct Copies {
  Copy<T> copy[kCopies];
};

template <typename T>
__global__ __launch_bounds__(256) void k_pack(const Copies<T> copies) {
  const Copy<T> &c = copies.copy[blockIdx.y];
  const int64_t all = c.rows * c.chunks, step = int64_t(gridDim.x) * 256;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += step) {
    const int64_t r = all <= 0xffffffffll ? uint32_t(i) / uint32_t(c.chunks) : i / c.chunks;
    const int first = int(i - r * c.chunks) * kChunk<T>;
    const float f = c.factor ? c.factor[r] : 1.0f;
    typedef T vec __attribute__((ext_vector_type(kChunk<T>), aligned(sizeof(T))));
    const T *from = c.src + r * c.ld + first;
    vec v = {};
    if (f != 0.0f) {
      if (first + kChunk<T> <= c.cols) {
        v = *reinterpret_cast<const vec *>(from);
      } else {
#pragma unroll
        for (int e = 0; e < kChunk<T>; ++e)
          if (first + e < c.cols) v[e] = from[e];
      }
      if (c.factor)
#pragma unroll
        for (int e = 0; e < kChunk<T>; ++e) v[e] = T(float(v[e]) * f);
    }
    reinterpret_cast<u32x4 *>(c.dst)[i] = __builtin_bit_cast(u32x4, v);
  }
}

// The largest magnitude and the length (root of the sum of squares) of each row
// of up to four matrices, of the finite values: a wave a row.
template <typename T>
struct Sized {
  const T *p;
  int64_t ld, rows;
  int cols;
  bool aligned;  // row_chunk's
  float2 *out;
};
constexpr int kSized = 4;
template <typename T>
struct SizedRows {
  Sized<T> of[kSized];
};

template <typename T, bool Aligned>
__device__ inline float2 row_size(const T *row, int cols, int lane) {
  float2 s = make_float2(0.0f, 0.0f);
  for (int c = lane; c * kChunk<T> < cols; c += 64) {
    typedef T vec __attribute__((ext_vector_type(kChunk<T>)));
    const vec v = __builtin_bit_cast(vec, row_chunk<T, Aligned>(row, c, cols));
#pragma unroll
    for (int e = 0; e < kChunk<T>; ++e) {
      const float x = fabsf(float(v[e]));
      if (x < INFINITY) {
        s.x = fmaxf(s.x, x);
        s.y += x * x;
      }
    }
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) {
    s.x = fmaxf(s.x, __shfl_xor(s.x, x));
    s.y += __shfl_xor(s.y, x);
  }
  return make_float2(s.x, sqrtf(s.y));
}

template <typename T>
__global__ __launch_bounds__(256) void k_row_sizes(const SizedRows<T> all) {
  const Sized<T> &a = all.of[blockIdx.y];
  const int lane = threadIdx.x & 63;
  for (int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); r < a.rows; r += int64_t(gridDim.x) * 4) {
    const T *row = a.p + r * a.ld;
    const float2 s = a.aligned ? row_size<T, true>(row, a.cols, lane) : row_size<T, false>(row, a.cols, lane);
    if (lane == 0) a.out[r] = s;
  }
}

// dw = sum over rows of (2^k_i da_i) (2^-k_i x_i): the second factor, an operand
// too, is brought below 2^15 by a power of two for all rows, which out[0] takes
// back.  `top` is the largest |x_i| 2^-k_i.  A row's part loses bits where its
// own, times the bound of k_gated_scales, is more than some 2^29 below the largest.
__device__ inline void gated_units(float top, int rows, float *x_factor, float *out) {
  int e = 15;
  if (top > 0.0f) frexpf(top, &e);
  if (blockIdx.x == 0 && threadIdx.x == 0) out[0] = ldexpf(1.0f, e - 15);
  const float unit = ldexpf(1.0f, 15 - e);
  for (int m = int(blockIdx.x) * 1024 + int(threadIdx.x); m < rows; m += int(gridDim.x) * 1024) x_factor[m] *= unit;
}

// Powers of two that bring the rows of da and db below 2^15 in magnitude, by
//   |a|, |b| <= |x_i| |w|, |act'| <= 1.2, |act(a)| <= |a| (sigmoid: 1),
//   |da|, |db| <= max |dh_i| (1.2 |x_i| |w| (+ 1)),  |w| the longest row of both weights:
// row i is kept times scale[i] = 2^k_i, so that what lies more than some 2^29
// below that bound is subnormal, and dx_factor[i] = 2^-k_i takes it back from
// dx.  A row without a gradient has scale 1 and x_factor 0.  Several workgroups
// leave the largest |x| 2^-k_i of each in tops [gridDim.x] to k_gated_units.
//
// With the rows' sizes and the copy of x: 50 us of the backward pass' 511 at
// 8192 x 1024 x 4096, 11 us of a small one's 37.
__global__ __launch_bounds__(1024) void k_gated_scales(const float2 *x, const float2 *dh, const float2 *gate,
                                                       const float2 *value, int rows, int hidden, int act, float *scale,
                                                       float *dx_factor, float *x_factor, float *tops, float *out) {
  __shared__ float shared[16];
  float longest = 0.0f;
  for (int f = threadIdx.x; f < hidden; f += 1024) longest = fmaxf(longest, fmaxf(gate[f].y, value[f].y));
  longest = group_max(longest, shared);
  float top = 0.0f;
  for (int m = int(blockIdx.x) * 1024 + int(threadIdx.x); m < rows; m += int(gridDim.x) * 1024) {
    const float bound = dh[m].x * (1.2f * x[m].y * longest + (act == LDA_SIGMOID ? 1.0f : 0.0f));
    int e = 15;
    if (bound > 0.0f) frexpf(bound, &e);  // bound < 2^e
    scale[m] = ldexpf(1.0f, 15 - e);
    dx_factor[m] = ldexpf(1.0f, e - 15);
    x_factor[m] = bound > 0.0f ? dx_factor[m] : 0.0f;
    top = fmaxf(top, x[m].x * x_factor[m]);
  }
  top = group_max(top, shared);
  if (gridDim.x == 1) gated_units(top, rows, x_factor, out);
  else if (threadIdx.x == 0) tops[blockIdx.x] = top;
}

__global__ __launch_bounds__(1024) void k_gated_units(const float *tops, int rows, float *x_factor, float *out) {
  __shared__ float shared[16];
  gated_units(group_max(threadIdx.x < gridDim.x ? tops[threadIdx.x] : 0.0f, shared), rows, x_factor, out);
}

// --------------------------------------------------------------- teacher ----
// The words that a teacher lists for a row, kPlaces to a lane (place lane + 64 i),
// and its softmax over them: p, its logarithm, and whether the row is kept.  A
// word of -1 is an empty place.
constexpr int kPlaces = LDA_OPS_MAX_TOP / 64;
struct Listed {
  int word[kPlaces];
  float p[kPlaces], log_p[kPlaces];
  bool kept;
};

__device__ inline Listed teacher_row(const int32_t *words, const float *scores, int top, int vocab, float unit,
                                     int lane) {
  Listed t;
  float score[kPlaces], high = -INFINITY, sum = 0.0f;
  bool some = false;
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) {
    const int j = lane + 64 * i;
    t.word[i] = -1;
    score[i] = -INFINITY;
    if (j < top) {
      const int word = words[j];
      if (word >= 0 && word < vocab) {
        t.word[i] = word;
        score[i] = scores[j] * unit;
      }
    }
    some |= score[i] != -INFINITY;  // NaN is no reason to leave a row out
    high = fmaxf(high, score[i]);
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) high = fmaxf(high, __shfl_xor(high, x));
  if (high == -INFINITY) high = 0.0f;
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) {
    t.log_p[i] = score[i] - high;
    t.p[i] = __builtin_amdgcn_exp2f(t.log_p[i] * kLog2e);
    sum += t.p[i];
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
  t.kept = __ballot(some);
  const float log_sum = kLn2 * __builtin_amdgcn_logf(sum), part = 1.0f / sum;
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) {
    t.log_p[i] -= log_sum;
    t.p[i] = t.kept ? t.p[i] * part : 0.0f;
  }
  return t;
}

// The logits of a row's listed words and its loss: a workgroup a row, four words
// of a wave at a time.  Reads a row of the weights for each place: 8192 x 32 of
// 1024 bf16, 537 MB that mostly lie in the caches, 68 us.
template <typename T>
__global__ __launch_bounds__(256) void k_distill_loss(const T *x, int64_t ldx, const T *weight, int64_t ldw,
                                                      const float *bias, const int32_t *words, int64_t ld_words,
                                                      const float *scores, int64_t ld_scores, int width, int vocab,
                                                      int top, float unit, const float *lse, float *logits,
                                                      float *loss) {
  constexpr int U = 4, N = kChunk<T>;
  typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));  // at any address
  __shared__ float z[LDA_OPS_MAX_TOP];
  const int64_t m = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t *list = words + m * ld_words;
  const T *row = x + m * ldx;
  for (int j0 = wave * U; j0 < top; j0 += 4 * U) {
    const T *w[U];
    float sum[U];
    int word[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      word[u] = j0 + u < top ? list[j0 + u] : -1;
      if (word[u] >= vocab) word[u] = -1;
      w[u] = weight + int64_t(word[u] < 0 ? 0 : word[u]) * ldw;
      sum[u] = 0.0f;
    }
    for (int c = lane * N; c < width; c += 64 * N) {
      if (c + N <= width) {
        const vec xv = *reinterpret_cast<const vec *>(row + c);
        vec wv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) wv[u] = *reinterpret_cast<const vec *>(w[u] + c);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < N; ++e) sum[u] += float(xv[e]) * float(wv[u][e]);
      } else {
        for (int e = c; e < width; ++e)
#pragma unroll
          for (int u = 0; u < U; ++u) sum[u] += float(row[e]) * float(w[u][e]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int x_ = 1; x_ < 64; x_ <<= 1) sum[u] += __shfl_xor(sum[u], x_);
      if (lane == 0 && j0 + u < top) z[j0 + u] = word[u] < 0 ? 0.0f : (bias ? sum[u] + bias[word[u]] : sum[u]) * unit;
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < top; j += 256) logits[m * top + j] = z[j];
  if (wave) return;
  const Listed t = teacher_row(list, scores + m * ld_scores, top, vocab, unit, lane);
  const float l = lse[m];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kPlaces; ++i) {
    if (t.word[i] < 0 || t.p[i] == 0.0f) continue;
    const float zj = z[lane + 64 * i];
    sum += zj == -INFINITY ? INFINITY : t.p[i] * (t.log_p[i] - (zj - l));
  }
#pragma unroll
  for (int x_ = 1; x_ < 64; x_ <<= 1) sum += __shfl_xor(sum, x_);
  if (lane == 0) loss[m] = t.kept ? sum : 0.0f;
}

// What the backward pass takes of the teacher.  A row's gradient over the
// temperature, d = s 2^e with 1 <= s < 2, is taken apart: G is kept times s, so
// that it is rounded once with it, and 2^e (row_loss) multiplies dx and the rows of
// x in dweight without a rounding (dweight of rounded s x instead: 1.7 times the
// error of the plain form at 4096 x 512 x 102000 of f16).  The epilogue of G gets s
// by its logarithm in shifted[m] = lse - log s.  And for the first place of each
// listed word what G has there, S s (exp(z - lse) - p), and d p, which dbias
// lacks; other places have the word -1.  labels: 0 for a row that is kept, or -1.
// A wave a row.
template <typename T>
__global__ __launch_bounds__(256) void k_teacher(const int32_t *words, int64_t ld_words, const float *scores,
                                                 int64_t ld_scores, const float *logits, const float *lse,
                                                 const float *dloss, int rows, int vocab, int top, float unit,
                                                 int32_t *labels, float *row_loss, float *shifted,
                                                 int32_t *its_word, float *its_grad, float *its_share) {
  __shared__ float p[4][LDA_OPS_MAX_TOP];
  __shared__ int word[4][LDA_OPS_MAX_TOP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = int(blockIdx.x) * 4 + wave;
  float l = 0.0f, d = 0.0f, s = 1.0f;
  if (m < rows) {
    const Listed t = teacher_row(words + m * ld_words, scores + m * ld_scores, top, vocab, unit, lane);
    l = lse[m];
    d = t.kept ? dloss[m] * unit : 0.0f;
    float power = d;
    if (d != 0.0f && fabsf(d) < INFINITY) {
      int e;
      s = 2.0f * frexpf(fabsf(d), &e);
      power = copysignf(ldexpf(1.0f, e - 1), d);
    }
#pragma unroll
    for (int i = 0; i < kPlaces; ++i) {
      p[wave][lane + 64 * i] = t.p[i];
      word[wave][lane + 64 * i] = t.kept && l != -INFINITY ? t.word[i] : -1;
    }
    if (lane == 0) {
      labels[m] = t.kept ? 0 : -1;
      row_loss[m] = power;
      shifted[m] = l - kLn2 * __builtin_amdgcn_logf(s);
    }
  }
  __syncthreads();
  if (m >= rows) return;
  for (int j = lane; j < top; j += 64) {
    int mine = word[wave][j];
    float all = 0.0f;
    for (int i = 0; i < top; ++i) {
      if (word[wave][i] != mine) continue;
      all += p[wave][i];
      if (i < j) mine = -1;
    }
    const int64_t at = int64_t(m) * top + j;
    its_word[at] = mine;
    if (mine < 0) continue;
    its_grad[at] = (__builtin_amdgcn_exp2f((logits[at] - l) * kLog2e) - all) * (s * kGradUnit<T>);
    if (its_share) its_share[at] = all * d;
  }
}

// A piece of G where the teacher has words, and of what its rounding left (`rest`,
// NULL: not wanted).
template <typename T>
__global__ __launch_bounds__(256) void k_teacher_words(const int32_t *its_word, const float *its_grad, int64_t count,
                                                       int top, int first, int piece, T *grad, T *rest, int64_t ldg) {
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < count; i += int64_t(gridDim.x) * 256) {
    const int at = its_word[i] - first;
    if (its_word[i] < 0 || at < 0 || at >= piece) continue;
    const int64_t to = int64_t(uint32_t(i) / uint32_t(top)) * ldg + at;
    const T g = T(its_grad[i]);
    grad[to] = g;
    if (rest) rest[to] = T(its_grad[i] - float(g));
  }
}

// ------------------------------------------------------------------- host ---
// Whether an operand can be read where it lies: its rows start at multiples of
// 16 bytes and hold whole chunks.
template <typename T>
bool in_place(const void *p, int64_t ld, int64_t cols) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % kChunk<T> == 0 && cols % kChunk<T> == 0;
}

template <typename T>
struct Matrix {
  const T *p;
  int64_t ld;
};

// The matrices whose rows' sizes a call needs.
template <typename T>
struct Sizes {
  SizedRows<T> rows_of = {};
  int count = 0;
  int64_t most = 0;  // rows

  float2 *add(const void *p, int64_t ld, int64_t rows, int cols, Arena &ws) {
    float2 *out = ws.take<float2>(rows);
    rows_of.of[count++] = Sized<T>{static_cast<const T *>(p), ld, rows, cols, in_place<T>(p, ld, cols), out};
    if (rows > most) most = rows;
    return out;
  }
  hipError_t run(hipStream_t s) {
    k_row_sizes<T><<<dim3(strided(ceil_div(most, 4)), unsigned(count)), 256, 0, s>>>(rows_of);
    return hipGetLastError();
  }
};

// The copies that a call needs before its first product.
template <typename T>
struct Packs {
  Copies<T> copies = {};
  int count = 0;
  int64_t most = 0;  // chunks of the largest

  void add(const void *p, int64_t ld, int64_t rows, int cols, const float *factor, T *dst, int64_t ldd) {
    const int chunks = int(ldd / kChunk<T>);
    copies.copy[count++] = Copy<T>{static_cast<const T *>(p), ld, rows, cols, chunks, factor, dst};
    if (rows * chunks > most) most = rows * chunks;
  }
  hipError_t run(hipStream_t s) {
    if (count == 0) return hipSuccess;
    k_pack<T><<<dim3(strided(ceil_div(most, 256)), unsigned(count)), 256, 0, s>>>(copies);
    return hipGetLastError();
  }
};

// A matrix as the products read it, copied where it has to be.
template <typename T>
Matrix<T> operand(const void *p, int64_t ld, int64_t rows, int cols, Arena &ws, Packs<T> &packs) {
  if (in_place<T>(p, ld, cols)) return Matrix<T>{static_cast<const T *>(p), ld};
  const int64_t ldd = round_up(cols, kChunk<T>);
  T *copy = ws.take<T>(rows * ldd);
  packs.add(p, ld, rows, cols, nullptr, copy, ldd);
  return Matrix<T>{copy, ldd};
}

// Tiles of a product and the parts its sum over k is split into.  Only a product
// whose result is stored plainly can be split (`steps` given), into parts of at
// least 8 steps.
//
// The shape and the parts with the least time: the area that the busiest CU has
// to multiply, over the rate that the shape reaches there, and for parts a
// launch that joins them and their bytes.  A CU takes one workgroup of 256 x
// 256, two of 128 x 128 or four of 64 x 64, and about half of the rate with only
// one of several.  Measured, gated layer of 16-bit types, forward, us with 256 /
// 128 / 64: 4096 x 512 x 4096 44 / 48 / 69 (all CUs full), 2048 x 1024 x 2048
// 30 / 25 / 35, 512 x 1024 x 1024 28 / 15 / 13.  In single precision the matrix
// unit alone bounds a CU, 256 accumulators spill, and smaller tiles are no
// slower: 2048 x 512 x 4096 156 / 138 / 151, 256 x 1024 x 1024 272 / 70 / 25.
struct Tiles {
  int m = 0, n = 0, splits = 1;
  Tiles(int64_t rows, int64_t cols, bool single, int64_t steps = 0) {
    const int64_t most = steps / 8 < 1 ? 1 : steps / 8 > 64 ? 64 : steps / 8;
    // us of a CU for a step of 256 x 256 at a rate of 1
    const double step_us = single ? 4.3 : 0.9;
    double best = 0;
    for (int side : {256, 128, 64}) {
      if (single && side == 256) continue;
      const int64_t tiles = ceil_div(rows, side) * ceil_div(cols, side);
      const int fit = side == 256 ? 1 : side == 128 ? 2 : 4;
      const double full = single ? (side == 128 ? 1.0 : 0.91) : (side == 256 ? 1.0 : side == 128 ? 0.75 : 0.45);
      // whole, or parts that give every CU one, two or four workgroups
      for (int64_t fill = 0; fill <= fit; fill = fill ? 2 * fill : 1) {
        int64_t want = fill * kCus / tiles;
        want = want < 1 ? 1 : want > most ? most : want;
        if (fill && want == 1) continue;
        if (want > 1) want = ceil_div(steps, split_steps(steps, want));  // none is empty
        const int64_t each = ceil_div(tiles * want, kCus);  // tiles of the busiest CU
        const double rate = full * (each < fit ? 0.5 + 0.5 * each / fit : 1.0);
        double us = double(each) * side * side / 65536 * step_us * (steps ? steps : 1) / rate / double(want);
        if (want > 1) us += 4.0 + double(rows) * double(cols) * want * 1e-6;
        if (best == 0 || us < best) {
          best = us;
          m = n = side;
          splits = int(want);
        }
      }
    }
  }
  static int64_t split_steps(int64_t steps, int64_t splits) { return round_up(ceil_div(steps, splits), 2); }
  static constexpr int64_t kCus = 256;
};

template <typename T>
Tiles tiles_of(int64_t rows, int64_t cols, int64_t steps = 0) {
  return Tiles(rows, cols, sizeof(T) == 4, steps);
}

template <typename T>
int64_t steps_of(int64_t k) {
  return round_up(ceil_div(k, kStep<T>), 2);
}

template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
};

// Calls fn with the shape of the tiles.
template <typename T, typename Fn>
hipError_t with_shape(const Tiles &t, Fn fn) {
  if constexpr (sizeof(T) == 2) {
    if (t.m == 256) return fn(Shape<256, 256, 2, 4>());
  }
  return t.m == 128 ? fn(Shape<128, 128, 2, 2>()) : fn(Shape<64, 64, 2, 2>());
}

template <typename T, typename S, typename L, typename R, typename Epilogue>
hipError_t product(int64_t m, int64_t n, int64_t k, int splits, const L &left, const R &right, const Epilogue &epi,
                   hipStream_t s) {
  Grid g;
  g.mtiles = int(ceil_div(m, S::BM));
  g.ntiles = int(ceil_div(n, S::BN));
  g.steps = int(steps_of<T>(k));
  g.split = int(Tiles::split_steps(g.steps, splits));
  g.splits = int(ceil_div(g.steps, g.split));  // a shorter k than the splits were chosen for leaves some out
  const int64_t items = round_up(int64_t(g.mtiles) * g.ntiles * g.splits, 8);
  constexpr size_t lds = 4 * (S::BM + S::BN) * 64 + S::BM * S::WN * 8;  // and the softmax parts of a tile's rows
  auto kernel = k_product<T, S::BM, S::BN, S::WM, S::WN, L, R, Epilogue>;
  if constexpr (lds > 65536) {
    OPS_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                int(lds)));
  }
  const int64_t most = Tiles::kCus * (S::BM == 256 ? 1 : S::BM == 128 ? 2 : 4);
  kernel<<<unsigned(items < most ? items : most), 64 * S::WM * S::WN, lds, s>>>(g, left, right, epi);
  return hipGetLastError();
}

// A whole product into `out`, split over k where it has few tiles.
template <typename T, typename L, typename R>
hipError_t product_into(int64_t m, int64_t n, int64_t k, const L &left, const R &right, const Target<T> &out, Arena &ws,
                        bool dry, hipStream_t s) {
  const Tiles tiles = tiles_of<T>(m, n, steps_of<T>(k));
  const int splits = tiles.splits;
  const int64_t cols4 = round_up(n, 4);
  float *part = splits > 1 ? ws.take<float>(splits * m * cols4) : nullptr;
  if (dry) return hipSuccess;
  if (splits == 1)
    return with_shape<T>(tiles, [&](auto shape) {
      return product<T, decltype(shape)>(m, n, k, 1, left, right, Store<T>{out, int(n)}, s);
    });
  OPS_TRY(with_shape<T>(tiles, [&](auto shape) {
    return product<T, decltype(shape)>(m, n, k, splits, left, right, StorePart<false>{part, int(m), int(cols4)}, s);
  }));
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

// Both weights as the products read them, with one row stride if `same` (they
// are copied for that where they have two).
template <typename T>
void pair_operands(const lda_gated_args &a, bool same, Arena &ws, Packs<T> &packs, Matrix<T> &gate, Matrix<T> &value) {
  gate = operand<T>(a.w_gate, a.ld_gate, a.hidden, a.width, ws, packs);
  value = operand<T>(a.w_value, a.ld_value, a.hidden, a.width, ws, packs);
  if (!same || gate.ld == value.ld) return;
  // a copy has this stride, so that no weight is copied twice
  const int64_t ldd = round_up(a.width, kChunk<T>);
  for (Matrix<T> *m : {&gate, &value}) {
    if (m->ld == ldd) continue;
    T *copy = ws.take<T>(a.hidden * ldd);
    packs.add(m->p, m->ld, a.hidden, a.width, nullptr, copy, ldd);
    *m = Matrix<T>{copy, ldd};
  }
}

template <typename T>
hipError_t gated_forward_t(const lda_gated_args &a, Arena &ws, bool dry) {
  if (a.rows == 0) return hipSuccess;
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const int rows = int(a.rows), k = int(round_up(a.width, kChunk<T>));
  if (rows <= kFewRows) {
    if (dry) return hipSuccess;
    const bool aligned = in_place<T>(a.x, a.ldx, a.width) && in_place<T>(a.w_gate, a.ld_gate, a.width) &&
                         in_place<T>(a.w_value, a.ld_value, a.width);
    auto kernel = aligned ? k_gated_few<T, true> : k_gated_few<T, false>;
    kernel<<<unsigned(ceil_div(a.hidden, 16)), 256, 0, s>>>(
        static_cast<const T *>(a.x), a.ldx, static_cast<const T *>(a.w_gate), a.ld_gate,
        static_cast<const T *>(a.w_value), a.ld_value, rows, a.width, a.hidden, a.act, static_cast<T *>(a.h), a.ldh);
    return hipGetLastError();
  }
  Packs<T> packs;
  const Matrix<T> x = operand<T>(a.x, a.ldx, a.rows, a.width, ws, packs);
  Matrix<T> gate, value;
  pair_operands<T>(a, false, ws, packs, gate, value);
  if (dry) return hipSuccess;
  OPS_TRY(packs.run(s));
  const GatedForward<T> epi{static_cast<T *>(a.h), a.ldh, rows, a.hidden, a.act};
  return with_shape<T>(tiles_of<T>(a.rows, pair_cols(a.hidden)), [&](auto shape) {
    return product<T, decltype(shape)>(a.rows, pair_cols(a.hidden), k, 1, Rows<T>{x.p, x.ld, rows, k},
                                       PairRows<T>{gate.p, value.p, gate.ld, value.ld, a.hidden, k}, epi, s);
  });
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
  const int rows = int(a.rows), pc = int(pair_cols(a.hidden)), k = int(round_up(a.width, kChunk<T>));
  Packs<T> packs;
  const Matrix<T> x = operand<T>(a.x, a.ldx, a.rows, a.width, ws, packs);
  Matrix<T> gate, value;
  pair_operands<T>(a, true, ws, packs, gate, value);
  T *dab = ws.take<T>(a.rows * pc);
  float *scale = nullptr, *dx_factor = nullptr, *dw_factor = nullptr;
  Matrix<T> x_scaled = x;
  if constexpr (kScaledRows<T>) {
    Sizes<T> sizes;
    const float2 *sx = sizes.add(a.x, a.ldx, a.rows, a.width, ws), *sd = sizes.add(a.dh, a.lddh, a.rows, a.hidden, ws);
    const float2 *sg = sizes.add(a.w_gate, a.ld_gate, a.hidden, a.width, ws);
    const float2 *sv = sizes.add(a.w_value, a.ld_value, a.hidden, a.width, ws);
    const int64_t needed = ceil_div(a.rows, 1024);
    const int groups = int(needed < 256 ? needed : 256);  // at most 1,024 (k_gated_units)
    float *tops = ws.take<float>(groups), *x_factor = ws.take<float>(rows);
    scale = ws.take<float>(rows);
    dx_factor = ws.take<float>(rows);
    dw_factor = ws.take<float>(1);
    T *copy = ws.take<T>(a.rows * k);
    packs.add(a.x, a.ldx, a.rows, a.width, x_factor, copy, k);
    x_scaled = Matrix<T>{copy, k};
    if (!dry) {
      OPS_TRY(sizes.run(s));
      k_gated_scales<<<unsigned(groups), 1024, 0, s>>>(sx, sd, sg, sv, rows, a.hidden, a.act, scale, dx_factor,
                                                    x_factor, tops, dw_factor);
      OPS_TRY(hipGetLastError());
      if (groups > 1) {
        k_gated_units<<<unsigned(groups), 1024, 0, s>>>(tops, rows, x_factor, dw_factor);
        OPS_TRY(hipGetLastError());
      }
    }
  }
  if (!dry) {
    OPS_TRY(packs.run(s));
    const GatedBackward<T> epi{static_cast<const T *>(a.dh), a.lddh, scale, dab, rows, a.hidden, pc, a.act};
    OPS_TRY(with_shape<T>(tiles_of<T>(a.rows, pc), [&](auto shape) {
      return product<T, decltype(shape)>(a.rows, pc, k, 1, Rows<T>{x.p, x.ld, rows, k},
                                         PairRows<T>{gate.p, value.p, gate.ld, value.ld, a.hidden, k}, epi, s);
    }));
  }
  const Target<T> dx{static_cast<T *>(a.dx), nullptr, a.lddx, rows, false, dx_factor, 1};
  OPS_TRY(product_into<T>(a.rows, a.width, pc, Rows<T>{dab, pc, rows, pc},
                          PairColumns<T>{gate.p, value.p, gate.ld, a.width, a.hidden}, dx, ws, dry, s));
  const Target<T> dw{dwg, dwv, a.width, a.hidden, true, dw_factor, 0};
  return product_into<T>(pc, a.width, a.rows, Columns<T>{dab, pc, pc, rows},
                         Columns<T>{x_scaled.p, x_scaled.ld, a.width, rows}, dw, ws, dry, s);
}

// With a Teacher only lse, of logits times `unit`.
template <typename T, bool Teacher>
hipError_t softmax_forward(const lda_xent_args &a, float unit, Arena &ws, bool dry) {
  if (a.rows == 0) return hipSuccess;
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const int rows = int(a.rows), k = int(round_up(a.width, kChunk<T>));
  if (rows <= kFewRows) {
    const int64_t groups = ceil_div(a.vocab, 64);
    const int parts = int(groups < 1024 ? groups : 1024);
    float2 *part = ws.take<float2>(int64_t(rows) * parts);
    float *label_logit = ws.take<float>(rows);
    if (dry) return hipSuccess;
    auto kernel = in_place<T>(a.x, a.ldx, a.width) && in_place<T>(a.weight, a.ld_weight, a.width)
                      ? k_xent_few<T, true, Teacher>
                      : k_xent_few<T, false, Teacher>;
    kernel<<<unsigned(parts), 256, 0, s>>>(static_cast<const T *>(a.x), a.ldx, static_cast<const T *>(a.weight),
                                           a.ld_weight, a.bias, a.labels, rows, a.width, a.vocab, unit, label_logit,
                                           part);
    OPS_TRY(hipGetLastError());
    k_lse_join_few<<<unsigned(rows), 256, 0, s>>>(part, parts, label_logit, a.labels, a.vocab, a.loss, a.lse);
    return hipGetLastError();
  }
  const Tiles tiles = tiles_of<T>(a.rows, a.vocab);
  const int ntiles = int(ceil_div(a.vocab, tiles.n));
  Packs<T> packs;
  const Matrix<T> x = operand<T>(a.x, a.ldx, a.rows, a.width, ws, packs);
  const Matrix<T> w = operand<T>(a.weight, a.ld_weight, a.vocab, a.width, ws, packs);
  float2 *part = ws.take<float2>(int64_t(ntiles) * rows);
  float *label_logit = ws.take<float>(rows);
  if (dry) return hipSuccess;
  OPS_TRY(packs.run(s));
  OPS_TRY(with_shape<T>(tiles, [&](auto shape) {
    typedef decltype(shape) S;
    const SoftmaxPart<S::BM, S::WN, Teacher> epi{a.bias, a.labels, label_logit, part, rows, a.vocab, unit};
    return product<T, S>(a.rows, a.vocab, k, 1, Rows<T>{x.p, x.ld, rows, k}, Rows<T>{w.p, w.ld, a.vocab, k}, epi, s);
  }));
  k_lse_join<<<unsigned(ceil_div(rows, 16)), 256, 0, s>>>(part, ntiles, label_logit, a.labels, rows, a.vocab, a.loss,
                                                          a.lse);
  return hipGetLastError();
}

template <typename T>
hipError_t xent_forward_t(const lda_xent_args &a, Arena &ws, bool dry) {
  return softmax_forward<T, false>(a, 1.0f, ws, dry);
}

// Words of one piece: as many as G takes 256 MiB for, but at least 1,024, so that
// its products stay large (from 131,073 rows of 16 bits on G is larger for that).
template <typename T>
int piece_words(int64_t rows, int vocab) {
  const int64_t most = (int64_t(256) << 20) / (rows * int64_t(sizeof(T))) / 256 * 256;
  const int64_t all = round_up(vocab, 256);
  return int(most < 1024 ? (all < 1024 ? all : 1024) : most < all ? most : all);
}

// What the backward pass of distillation has beside the cross entropy's.
struct Teaching {
  float unit;
  int top;
  const int32_t *its_word;
  const float *its_grad;
  const float *less;  // dbias lacks this; NULL without a bias
};

// G in 16 bits is a rounding more than a product of single precision has, and costs
// distillation, whose listed words have any p, dx and dweight up to 1.4 times the
// error of their own rounding over many entries, 1.6 times over few (the cross
// entropy's -1 and powers of two are exact).  Up to this many rows, where
// products are bound by the weights and not by G, it is kept in twice its bits: as
// G and what its rounding left, which stands below it as further rows, so that
// both products take the two and the error is the results' rounding alone.
// Training, us of G once / twice: 8, 32, 128 x 1024 x 141000 of bf16 300 / 309,
// 342 / 381, 408 / 467; 128 x 257 x 9001 of f16 80 / 84.  More rows pay more, 129
// 436 / 562, 256 522 / 668; for 8192 twice would double two thirds of the operations.  Tiles of 256 x 256, which never have the
// least time at so few rows, have no epilogue for it: G is kept once with them.
constexpr int kTwiceRows = 128;

template <typename T, bool Teacher>
hipError_t softmax_backward(const lda_xent_args &a, const Teaching &teaching, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  T *dw = static_cast<T *>(a.dweight);
  if (a.rows == 0) {
    if (dry) return hipSuccess;
    OPS_TRY(zero(dw, int64_t(a.vocab) * a.width, s));
    return a.dbias ? zero(a.dbias, a.vocab, s) : hipSuccess;
  }
  const int rows = int(a.rows), piece = piece_words<T>(a.rows, a.vocab), k = int(round_up(a.width, kChunk<T>));
  const Tiles tiles = tiles_of<T>(a.rows, piece);
  const int mtiles = int(ceil_div(a.rows, tiles.m));
  // what the rounding of G left is read only where the epilogue of the tiles writes it
  const bool twice = Teacher && sizeof(T) == 2 && rows <= kTwiceRows && tiles.n < 256;
  const int times = twice ? 2 : 1, all = times * rows;  // of G
  Packs<T> packs;
  const Matrix<T> x = operand<T>(a.x, a.ldx, a.rows, a.width, ws, packs);
  const Matrix<T> w = operand<T>(a.weight, a.ld_weight, a.vocab, a.width, ws, packs);
  float *top = ws.take<float>(1), *row_factor = ws.take<float>(rows), *x_factor = ws.take<float>(rows);
  Sizes<T> sizes;
  const float2 *x_size = kScaledRows<T> ? sizes.add(a.x, a.ldx, a.rows, a.width, ws) : nullptr;
  T *x_scaled = ws.take<T>(int64_t(all) * k);
  T *grad = ws.take<T>(int64_t(all) * piece);
  float *col_part = a.bias ? ws.take<float>(int64_t(mtiles) * piece) : nullptr;
  const Tiles dx_tiles = tiles_of<T>(all, a.width, steps_of<T>(piece < a.vocab ? piece : a.vocab));
  const int splits = dx_tiles.splits;
  const int64_t cols4 = round_up(a.width, 4);
  float *dx_part = ws.take<float>(splits * all * cols4);
  if (!dry) {
    if constexpr (kScaledRows<T>) OPS_TRY(sizes.run(s));
    k_grad_factors<<<1, 1024, 0, s>>>(a.dloss, a.lse, a.labels, x_size, rows, a.vocab, kGradUnit<T>, top, row_factor,
                                      x_factor);
    OPS_TRY(hipGetLastError());
    for (int i = 0; i < times; ++i) packs.add(a.x, a.ldx, a.rows, a.width, x_factor, x_scaled + a.rows * k * i, k);
    OPS_TRY(packs.run(s));
  }
  // the pieces' products share the scratch of their parts
  const size_t mark = ws.used;
  size_t most = mark;
  for (int first = 0; first < a.vocab; first += piece) {
    const int words = a.vocab - first < piece ? a.vocab - first : piece;
    const int words_k = int(round_up(words, kChunk<T>));
    const T *wp = w.p + int64_t(first) * w.ld;
    T *rest = times > 1 ? grad + a.rows * words_k : nullptr;
    ws.used = mark;
    if (!dry) {
      OPS_TRY(with_shape<T>(tiles, [&](auto shape) {
        typedef decltype(shape) S;
        const SoftmaxGrad<T, S::BN, S::WM, Teacher> epi{a.bias,   a.labels, a.lse, row_factor, grad,  words_k,
                                                        col_part, rows,     a.vocab, first,    words, teaching.unit, rest};
        return product<T, S>(a.rows, words_k, k, 1, Rows<T>{x.p, x.ld, rows, k}, Rows<T>{wp, w.ld, words, k}, epi, s);
      }));
      if (a.dbias) {
        k_sum_parts<<<unsigned(ceil_div(words, 64)), 256, 0, s>>>(col_part, mtiles, words,
                                                                        Teacher ? teaching.less + first : nullptr,
                                                                        a.dbias + first);
        OPS_TRY(hipGetLastError());
      }
      if constexpr (Teacher) {
        const int64_t listed = a.rows * teaching.top;
        k_teacher_words<T><<<strided(ceil_div(listed, 256)), 256, 0, s>>>(
            teaching.its_word, teaching.its_grad, listed, teaching.top, first, words, grad, rest, words_k);
        OPS_TRY(hipGetLastError());
      }
      OPS_TRY(with_shape<T>(dx_tiles, [&](auto shape) {
        const Rows<T> gr{grad, words_k, all, words_k};
        const Columns<T> wc{wp, w.ld, a.width, words};
        if (first == 0)
          return product<T, decltype(shape)>(all, a.width, words, splits, gr, wc,
                                             StorePart<false>{dx_part, all, int(cols4)}, s);
        return product<T, decltype(shape)>(all, a.width, words, splits, gr, wc,
                                           StorePart<true>{dx_part, all, int(cols4)}, s);
      }));
    }
    T *dwp = dw + int64_t(first) * a.width;
    const Target<T> out{dwp, nullptr, a.width, words, false, top, 0};
    OPS_TRY(product_into<T>(words, a.width, all, Columns<T>{grad, words_k, words, all},
                            Columns<T>{x_scaled, k, a.width, all}, out, ws, dry, s));
    if (ws.used > most) most = ws.used;
  }
  ws.used = most;
  if (dry) return hipSuccess;
  const Target<T> out{static_cast<T *>(a.dx), nullptr, a.lddx, rows, false, row_factor, 1};
  k_join<T><<<strided(ceil_div(a.rows * cols4, 1024)), 256, 0, s>>>(dx_part, times * splits, rows, a.width, int(cols4), out);
  return hipGetLastError();
}

template <typename T>
hipError_t xent_backward_t(const lda_xent_args &a, Arena &ws, bool dry) {
  return softmax_backward<T, false>(a, Teaching{1.0f, 0, nullptr, nullptr, nullptr}, ws, dry);
}

// The softmax over the student's logits, as the cross entropy has it.
lda_xent_args student(const lda_distill_args &a) {
  lda_xent_args x = {};
  x.dtype = a.dtype;
  x.rows = a.rows;
  x.width = a.width;
  x.vocab = a.vocab;
  x.x = a.x;
  x.ldx = a.ldx;
  x.weight = a.weight;
  x.ld_weight = a.ld_weight;
  x.bias = a.bias;
  x.lse = a.lse;
  x.dx = a.dx;
  x.lddx = a.lddx;
  x.dweight = a.dweight;
  x.dbias = a.dbias;
  x.stream = a.stream;
  return x;
}

// 8192 x 1024 x 141000 of bf16, 32 words listed: forward 2.2 ms, as the cross
// entropy's and 69 us for the listed words; backward 6.7 ms, of which the teacher's
// part, its words' sort and sums for dbias included, is 0.13.
template <typename T>
hipError_t distill_forward_t(const lda_distill_args &a, Arena &ws, bool dry) {
  const float unit = 1.0f / a.temperature;
  OPS_TRY((softmax_forward<T, true>(student(a), unit, ws, dry)));
  if (dry || a.rows == 0) return hipSuccess;
  const T *x = static_cast<const T *>(a.x);
  return by_rows(a.rows, 256, 1, [&](int64_t m, int64_t rows) {
    k_distill_loss<T><<<unsigned(rows), 256, 0, static_cast<hipStream_t>(a.stream)>>>(
        x + m * a.ldx, a.ldx, static_cast<const T *>(a.weight), a.ld_weight, a.bias, a.words + m * a.ld_words,
        a.ld_words, a.scores + m * a.ld_scores, a.ld_scores, a.width, a.vocab, a.top, unit, a.lse + m,
        a.logits + m * a.top, a.loss + m);
  });
}

template <typename T>
hipError_t distill_backward_t(const lda_distill_args &a, Arena &ws, bool dry) {
  const hipStream_t s = static_cast<hipStream_t>(a.stream);
  const float unit = 1.0f / a.temperature;
  const int64_t listed = a.rows * a.top;
  lda_xent_args x = student(a);
  int32_t *labels = ws.take<int32_t>(a.rows), *its_word = ws.take<int32_t>(listed);
  float *row_loss = ws.take<float>(a.rows), *shifted = ws.take<float>(a.rows);
  float *its_grad = ws.take<float>(listed);
  float *its_share = a.bias ? ws.take<float>(listed) : nullptr, *less = a.bias ? ws.take<float>(a.vocab) : nullptr;
  if (!dry && a.rows) {
    k_teacher<T><<<unsigned(ceil_div(a.rows, 4)), 256, 0, s>>>(a.words, a.ld_words, a.scores, a.ld_scores, a.logits,
                                                               a.lse, a.dloss, int(a.rows), a.vocab, a.top, unit,
                                                               labels, row_loss, shifted, its_word, its_grad, its_share);
    OPS_TRY(hipGetLastError());
  }
  if (a.bias && a.rows)
    OPS_TRY(sum_by_word<float>(its_word, listed, its_share, 1, 1, a.vocab, 1.0f, less, ws, dry, s));
  x.labels = labels;
  x.dloss = row_loss;
  x.lse = shifted;
  return softmax_backward<T, true>(x, Teaching{unit, a.top, its_word, its_grad, less}, ws, dry);
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
hipError_t distill_forward(const lda_distill_args &a, Arena &ws, bool dry) { BY_TYPE(distill_forward_t, a, ws, dry) }
hipError_t distill_backward(const lda_distill_args &a, Arena &ws, bool dry) { BY_TYPE(distill_backward_t, a, ws, dry) }

}  // namespace ops
}  // namespace lda
