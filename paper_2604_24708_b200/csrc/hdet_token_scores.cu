// Log probabilities of given tokens, entropies and the best alternatives, of hidden states against a large table, without keeping the
// logits (contract: include/hdet.h).  For each replica, with H the hidden states of its counted tokens and W its table:
//
//   Z = H W^T,  lse = log sum_v exp Z_v,  logprob = Z_y - lse,  entropy = lse - sum_v p_v Z_v,  the n_top largest Z_v
//
// One product of T x V x D, whose epilogue keeps of every row
//   M      its maximum, and n, how many classes have it
//   delta  sum of exp(z - M) over the others                 lse      = M + log n + log1p(delta / n)
//   U      sum of exp(z - M) (z - M) over them (<= 0)        logprob  = -((M - z_y) + log n + log1p(delta / n))
//                                                            entropy  = (log n + log1p(delta / n)) - U / (n + delta)
// Every term has one sign, so a log probability or an entropy near zero keeps its relative precision: nothing is 1 less a sum that
// holds the 1 (with lse and a plain sum a token of probability 1 - 1e-6 was several percent off).
//
//   pack     counted tokens move together (padding drops out)
//   scores   a CTA (or pair) takes 128 (256) tokens and a run of the vocabulary, tile by tile: a reader keeps its row's state and its
//            list of the best classes over the whole run
//            (or, where all logits together are few, leaves the logits and the largest of every 32)
//   join     a warp or a block a row: the runs' states and lists become the row's; the best are summed again in fp64 and ordered
// One or two tokens a replica take a kernel of their own in place of the first two (few).
#include <algorithm>
#include <climits>

#include "hdet_vocab.cuh"

namespace hdet {
namespace {

constexpr int kStageBytes = 2 * kOperandBytes;
// warp 0 copies, warp 1 issues the products, warps 4 - 11 read the accumulator: a quarter of its lanes (warp % 4) and half of its
// columns each
constexpr int kScoreThreads = 384, kFirstReader = 4, kReaders = 8, kReaderThreads = 32 * kReaders;
constexpr int kMaxStages = 6;
constexpr int kMargin = 4;                 // classes kept beyond n_top: as many could be out of order by the fp32 logits
constexpr int kMaxList = HDET_MAX_TOP + kMargin;
constexpr int kShort = 16, kLong = 32;     // a reader's list has one of these lengths
constexpr int kGroup = 8, kBuffer = 16;    // columns that are looked through at a time for a list; classes that wait to be put into it
static_assert(kMaxList <= kLong, "every list fits");
constexpr int kMaxSmem = 227 * 1024;
constexpr long long kSelftestLimitCycles = 4000000ll;   // 2 ms
constexpr int kChunk = 16;                 // steps of 64 that the tensor cores sum before fp32 additions take over, as in the loss

using Key = unsigned long long;            // a class in a list: falling order of its logit, then rising order of its id; 0: none

__device__ __forceinline__ Key key_of(float z, int v) {
  const unsigned u = __float_as_uint(z + 0.0f);            // -0 and 0 are equal
  return (Key)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (unsigned)~v;
}
__device__ __forceinline__ float logit_of(Key k) {
  const unsigned u = (unsigned)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int class_of(Key k) { return (int)~(unsigned)k; }

// 32 keys, one in each lane, into falling order; and the 32 largest of two such.
__device__ __forceinline__ Key exchange(Key k, int stride, bool larger) {
  const Key o = __shfl_xor_sync(0xffffffffu, k, stride);
  return larger == (k > o) ? k : o;
}
__device__ __forceinline__ float exchange(float x, int stride, bool larger);
template <typename T>
__device__ __forceinline__ T sorted(T k) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int stride = size / 2; stride > 0; stride /= 2) k = exchange(k, stride, ((lane & stride) == 0) == ((lane & size) == 0));
  return k;
}
template <typename T>
__device__ __forceinline__ T merged(T a, T b) {
  const int lane = threadIdx.x & 31;
  b = __shfl_sync(0xffffffffu, b, 31 - lane);
  T k = a > b ? a : b;
#pragma unroll
  for (int stride = 16; stride > 0; stride /= 2) k = exchange(k, stride, (lane & stride) == 0);
  return k;
}

// The same for 32 floats.
__device__ __forceinline__ float exchange(float x, int stride, bool larger) {
  const float o = __shfl_xor_sync(0xffffffffu, x, stride);
  return larger ? fmaxf(x, o) : fminf(x, o);
}

// The 32 largest of WARPS warps' sorted keys, in warp 0.  All threads of those warps; s: WARPS rows, free for the next use after a barrier.
template <int WARPS, typename T>
__device__ __forceinline__ T merged_of_warps(T mine, int warp, T (*s)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int half = WARPS / 2; half > 0; half /= 2) {
    if (warp >= half && warp < 2 * half) s[warp][lane] = mine;
    __syncthreads();
    if (warp < half) mine = merged(mine, s[warp + half][lane]);
  }
  return mine;
}

// A row's state over some of its classes.
struct State {
  float top, others, weighted, ties;       // M, delta, U, n
  __device__ __forceinline__ void clear() { top = -INFINITY; others = weighted = ties = 0.0f; }
  // Moves the reference up to `to` > top: those that had the maximum are others now.
  __device__ __forceinline__ void raise(float to) {
    const float d = top - to, f = exp_from(top, to), all = ties + others;
    if (all != 0.0f) {                     // (not for the first value, where top is -inf)
      weighted = f * fmaf(all, fmaxf(d, -1e4f), weighted);           // (where f is 0, so is that, however far apart the two are)
      others = f * all;
    }
    top = to;
    ties = 0.0f;
  }
  __device__ __forceinline__ void add(State o) {
    if (o.top > top) raise(o.top); else if (top > o.top) o.raise(top);
    others += o.others;
    weighted += o.weighted;
    ties += o.ties;
  }
  // A warp's logits, one in each lane (-inf: none), into a state that all lanes hold.
  __device__ __forceinline__ void add_warp(float z) {
    float most = z;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (most > top) raise(most);
    const bool is = z == top && z > -INFINITY;
    const float d = z - (top > -INFINITY ? top : 0.0f);
    float e = is ? 0.0f : exp2_fast(d * kLog2e);
    float u = e * fmaxf(d, -1e4f);                         // a logit of -inf adds 0, not NaN; one that is NaN makes others NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      e += __shfl_xor_sync(0xffffffffu, e, o);
      u += __shfl_xor_sync(0xffffffffu, u, o);
    }
    others += e;
    weighted += u;
    ties += (float)__popc(__ballot_sync(0xffffffffu, is));
  }
  // All of WARPS warps' lanes' states, in all of them.  Everything first moves to the common maximum.
  template <int WARPS>
  __device__ __forceinline__ void add_all(int warp, float (*s)[4]) {
    const int lane = threadIdx.x & 31;
    float most = top;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if constexpr (WARPS > 1) {
      if (lane == 0) s[warp][0] = most;
      __syncthreads();
      most = lane < WARPS ? s[lane][0] : -INFINITY;
#pragma unroll
      for (int o = WARPS / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      most = __shfl_sync(0xffffffffu, most, 0);
    }
    if (most > top) raise(most);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) add_sums(o);
    if constexpr (WARPS > 1) {
      if (lane == 0) { s[warp][1] = others; s[warp][2] = weighted; s[warp][3] = ties; }
      __syncthreads();
      others = lane < WARPS ? s[lane][1] : 0.0f;
      weighted = lane < WARPS ? s[lane][2] : 0.0f;
      ties = lane < WARPS ? s[lane][3] : 0.0f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) add_sums(o);
    }
  }
  __device__ __forceinline__ void add_sums(int o) {
    others += __shfl_xor_sync(0xffffffffu, others, o);
    weighted += __shfl_xor_sync(0xffffffffu, weighted, o);
    ties += __shfl_xor_sync(0xffffffffu, ties, o);
  }
};
static_assert(sizeof(State) == 16, "one store");

struct ScoreParams {
  CUtensorMap hidden, weight;
  int n_replicas, vocab, width, n_tokens;
  int rows_pad;             // rows per replica of everything packed
  bool weight_shared;
  const int* count;
  const int* target;        // -1: none given
  const int* token_of;
  float* z_target;
  State* part;              // scores: [job][half][row of the tile]; few: [replica][token][part]
  Key* lists;               // in falling order; scores: [job][half][entry][row of the tile]; few: [replica][token][part][entry]
  float* logits;            // kept: [replica][rows_pad][pitch], and the largest of every 32: [group][replica][rows_pad]
  float* group_top;
  int64_t pitch;
  int* floor;               // [replica][rows_pad]: some list of the row is full of logits from here on (ordered_bits)
  int n_parts;              // few: blocks a replica
  int n_units;              // of unit_of(CTAs) classes
  int list;                 // entries of a list that count, 0: none
  int held;                 // entries of a reader's list
  int clusters, most_jobs;  // that run at once; that there is room for
  int chunk, stages;
  Control* control;
  long long wait_limit;
  bool withhold;            // copies nothing, so that the waits run out (hdet_selftest_token_scores_wait)
  // join
  const __nv_bfloat16 *rows, *table;   // hidden states and table as join_kernel reads them
  int64_t rows_stride, rows_row, table_stride, table_row;
  bool rows_packed;         // rows are those of the counted tokens
  bool rows_vec;            // rows of both start on 16-byte boundaries
  ScoreOut out;
};

constexpr int kColumns = 32;               // that a reader takes at a time
// Classes that a run is made of.  A single CTA's tiles end with a box of 64 rows of the table: it is for few tokens, where every row that is
// copied without need counts (48 tokens x 50257, width 1024: 46.3 us, with 32 classes 48.0).
__host__ __device__ constexpr int unit_of(int ctas) { return 64 / ctas; }

// How many runs the vocabulary is cut into: every cluster takes equal jobs in turn, so the shortest end has the fewest rounds times the
// length of a run.  A narrow last tile counts as half of one (its copies of the hidden states are those of a whole one), and a run costs a
// tile more than its tiles (its start, and filling the lists).  A warp's lanes try different numbers; every warp of the launch finds the same.
// (Runs of whole tiles: 52.8 us for 3 x 777 tokens x 4099, width 520, which has 17 tiles for 8 runs.)
template <int CTAS>
__device__ __forceinline__ int splits_for(const ScoreParams& p, int row_tiles) {
  constexpr unsigned kTileUnits = 128 * CTAS / unit_of(CTAS);
  row_tiles = max(1, row_tiles);
  // many runs at once need no second round to even out; few take up to four
  const int lane = threadIdx.x & 31, at_once = p.clusters / row_tiles;
  const int most = min(p.n_units, max(1, min(p.most_jobs / row_tiles, at_once >= 16 ? at_once : 4 * at_once + 4)));
  Key best = ~0ull;
  for (int s = lane + 1; s <= most; s += 32) {
    const unsigned len = (p.n_units + s - 1) / s;
    if ((unsigned)s != (p.n_units + len - 1) / len) continue;            // the same length with fewer runs
    const unsigned rest = len % kTileUnits, tiles = len - rest + (rest ? max(rest, kTileUnits / 2) : 0);
    const unsigned rounds = ((unsigned)(row_tiles * s) + p.clusters - 1) / p.clusters;
    best = min(best, ((Key)rounds * (tiles + kTileUnits)) << 20 | (unsigned)s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
  return (int)(best & 0xfffffu);
}

constexpr int kNoList = 0, kKeep = -1;             // in the place of a list's length: no alternatives; the logits are kept
constexpr int kRowGroup = 32;

// ------------------------------------------------------------------------------------------------ lists
// The order of floats as that of integers (kNoFloor: that of -inf).
__device__ __forceinline__ int ordered_bits(float x) {
  const int u = __float_as_int(x);
  return u < 0 ? u ^ 0x7fffffff : u;
}
__device__ __forceinline__ float from_ordered(int u) { return __int_as_float(u < 0 ? u ^ 0x7fffffff : u); }

// A reader thread's list of its row's best classes, LENGTH of them in falling order, and behind it a buffer of classes on their way into
// it, both in shared memory (entry e of all threads lies together).  Putting a class into the list where it is found costs a warp as much as if
// all its rows had found one, and rows find theirs at different columns; so it goes into the buffer, and when some row's buffer is half
// full all rows put theirs in together: the buffer is sorted and merged with the list, by networks whose places are known to the compiler.
// (8 x 2048 tokens x 50257 classes, width 1024, without lists 1.16 ms.  With 12 entries, put in one at a time: 1.63 ms when found, 1.45 from the
// buffer.)
constexpr uint2 kNothing = {0xff800000u, 0u};      // a logit of -inf

// Brings the `wanted` best of n entries to the front, in order, equal ones by their ids: for the rare rows with equal logits where it matters.
__device__ __noinline__ void order_exactly(uint2* at, int n, int wanted) {
  for (int i = 0; i < wanted; ++i) {
    uint2 best = at[i * kReaderThreads];
    int place = i;
    for (int j = i + 1; j < n; ++j) {
      const uint2 u = at[j * kReaderThreads];
      const float a = __uint_as_float(u.x), b = __uint_as_float(best.x);
      if (a > b || (a == b && u.y < best.y)) {
        best = u;
        place = j;
      }
    }
    at[place * kReaderThreads] = at[i * kReaderThreads];
    at[i * kReaderThreads] = best;
  }
}

// Puts `waiting` classes of the buffer into the list; returns the logit of entry `list` - 1.  A call, since what it takes in registers and
// instructions would weigh on the loop that hardly ever comes here.
template <int LENGTH>
__device__ __noinline__ float empty_buffer(uint2* at, int waiting, int list) {
  float z[LENGTH], y[kBuffer];
  unsigned id[LENGTH], w[kBuffer];
#pragma unroll
  for (int e = 0; e < kBuffer; ++e) {
    const uint2 u = e < waiting ? at[(LENGTH + e) * kReaderThreads] : kNothing;
    y[e] = __uint_as_float(u.x);
    w[e] = u.y;
  }
#pragma unroll
  for (int e = 0; e < LENGTH; ++e) {
    const uint2 u = at[e * kReaderThreads];
    z[e] = __uint_as_float(u.x);
    id[e] = u.y;
  }
  const auto order = [](float& a, unsigned& i, float& b, unsigned& j) {     // a >= b
    const bool swap = b > a;
    const float more = fmaxf(a, b), less = fminf(a, b);
    const unsigned k = swap ? j : i, l = swap ? i : j;
    a = more; b = less; i = k; j = l;
  };
  // odd-even merge sort of the buffer
#pragma unroll
  for (int p = 1; p < kBuffer; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < kBuffer; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < kBuffer && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order(y[i + j], w[i + j], y[i + j + k], w[i + j + k]);
  // the LENGTH largest of both: the list's last against the buffer's first, and so on; then that (bitonic) sequence into order
  float out = -INFINITY;                           // the largest that fell out
#pragma unroll
  for (int e = 0; e < kBuffer; ++e) {
    order(z[LENGTH - 1 - e], id[LENGTH - 1 - e], y[e], w[e]);
    out = fmaxf(out, y[e]);
  }
#pragma unroll
  for (int k = LENGTH / 2; k >= 1; k /= 2)
#pragma unroll
    for (int e = 0; e < LENGTH; ++e)
      if ((e & k) == 0) order(z[e], id[e], z[e + k], id[e + k]);
  if (__any_sync(0xffffffffu, out == z[LENGTH - 1] && out > -INFINITY)) {
    for (int e = waiting; e < kBuffer; ++e) at[(LENGTH + e) * kReaderThreads] = kNothing;
    order_exactly(at, LENGTH + kBuffer, LENGTH);
  } else {
#pragma unroll
    for (int e = 0; e < LENGTH; ++e) at[e * kReaderThreads] = make_uint2(__float_as_uint(z[e]), id[e]);
  }
  float last = z[LENGTH - 1];
#pragma unroll
  for (int e = 0; e < LENGTH - 1; ++e)
    if (e == list - 1) last = z[e];
  return last;
}

template <int LENGTH>
struct List {
  uint2* at;                // this thread's first entry
  int waiting;              // in the buffer
  int size;                 // entries that count
  float above;              // a class has to have a larger logit: the list's last that counts, or what other lists of the row say
  __device__ __forceinline__ void clear(int row_floor) {
#pragma unroll
    for (int e = 0; e < LENGTH; ++e) at[e * kReaderThreads] = kNothing;
    waiting = 0;
    above = below(row_floor);
  }
  // The largest logit that a class below all of a full list has.  (One that equals the list's last may go before it, by its id.)
  static __device__ __forceinline__ float below(int row_floor) {
    return row_floor > kNoFloor ? from_ordered(row_floor == 0 ? -2 : row_floor - 1) : -INFINITY;      // -1 is -0, which equals 0
  }
  __device__ __forceinline__ void empty(int* row_floor) {
    const float last = empty_buffer<LENGTH>(at, waiting, size);
    waiting = 0;
    if (last > above) {
      above = last;
      atomicMax(row_floor, ordered_bits(above + 0.0f));
    }
    above = fmaxf(above, below(__ldcg(row_floor)));
  }
  // Columns v .. v + 7 of the row.
  __device__ __forceinline__ void look_through(const float* x, int v, int* row_floor) {
    if (__any_sync(0xffffffffu, waiting > kBuffer - kGroup)) empty(row_floor);
    uint2* to = at + (LENGTH + waiting) * kReaderThreads;
    const uint2* const from = to;
#pragma unroll
    for (int i = 0; i < kGroup; ++i)
      if (x[i] > above) {
        *to = make_uint2(__float_as_uint(x[i]), (unsigned)(v + i));
        to += kReaderThreads;
      }
    waiting += (int)(to - from) / kReaderThreads;
  }
  // At the run's end: the entries that count are in the order of their keys.
  __device__ __forceinline__ void finish(int* row_floor) {
    empty(row_floor);
    bool equal = false;
    for (int e = 0; e < min(size, LENGTH - 1); ++e) {
      const float z = __uint_as_float(at[e * kReaderThreads].x);
      equal = equal || (z > -INFINITY && z == __uint_as_float(at[(e + 1) * kReaderThreads].x));
    }
    if (__any_sync(0xffffffffu, equal)) order_exactly(at, LENGTH, size);
  }
};
template <>
struct List<kNoList> {
  uint2* at;
};
template <>
struct List<kKeep> {
  uint2* at;                // (not used)
  Rows rows;                // where the warp's rows of logits go
  uint32_t staging;
  int64_t group;            // this row's place in a group's maxima
};

// ------------------------------------------------------------------------------------------------ product
struct Shared {             // behind the stages and the lists
  uint64_t full[kMaxStages], empty[kMaxStages];    // a stage holds its operands; the products have read it
  uint64_t acc_full[2], acc_empty[2];              // an accumulator is complete; its readers are done with it
  uint32_t tmem;
  int failed;
  int count[HDET_MAX_REPLICAS];
  int splits;
};

constexpr int kStagingBytes = 4096;        // per reader: 32 rows x 128 bytes
__host__ __device__ constexpr int list_bytes(int held) {
  return held == kKeep ? kReaders * kStagingBytes : held ? 8 * (held + kBuffer) * kReaderThreads : 0;
}
constexpr int kFixedSmem = 1024 + (int)sizeof(Shared);
static_assert(kFixedSmem + 4 * kStageBytes + list_bytes(kLong) <= kMaxSmem, "four stages beside the longest lists");

struct Run {                // a cluster's job: 128 CTAS tokens of a replica, and classes from .. to (multiples of unit_of)
  int r, m0, from, to;
};

// A tile's columns, and the boxes of 64 rows of the table that a CTA copies for its share of them.
template <int CTAS>
__device__ __forceinline__ int columns_of(const Run& run, int n0) { return min(128 * CTAS, run.to - n0); }
template <int CTAS>
__device__ __forceinline__ int boxes_of(int columns) { return columns > 64 * CTAS ? 2 : 1; }

template <int CTAS>
__device__ __forceinline__ bool find_run(const ScoreParams& p, const Shared& sh, int job, Run& run) {
  constexpr int kTile = 128 * CTAS;
  const int splits = sh.splits, len = (p.n_units + splits - 1) / splits * unit_of(CTAS);
  // tokens fastest: runs that go on at the same time read the same rows of the table
  for (run.r = 0; run.r < p.n_replicas; ++run.r) {
    const int row_tiles = (sh.count[run.r] + kTile - 1) / kTile;
    if (job < row_tiles * splits) {
      run.m0 = job % row_tiles * kTile;
      run.from = job / row_tiles * len;
      run.to = min(run.from + len, p.n_units * unit_of(CTAS));
      // one value for the warp, so that what is worked out from it is the warp's too
      run.r = __shfl_sync(0xffffffffu, run.r, 0);
      run.m0 = __shfl_sync(0xffffffffu, run.m0, 0);
      run.from = __shfl_sync(0xffffffffu, run.from, 0);
      run.to = __shfl_sync(0xffffffffu, run.to, 0);
      return true;
    }
    job -= row_tiles * splits;
  }
  return false;
}

// 32 columns of a row, from class v on, into its state and list.
template <int LENGTH>
__device__ __forceinline__ void take_logits(const ScoreParams& p, float (&x)[32], int v, int target, int64_t row, State& s, List<LENGTH>& list) {
  if (v + 32 > p.vocab) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (v + i >= p.vocab) x[i] = -INFINITY;      // behind the vocabulary's end: nothing of theirs is left in exp
  }
  float most[32 / kGroup];
#pragma unroll
  for (int g = 0; g < 32 / kGroup; ++g) {
    most[g] = x[kGroup * g];
#pragma unroll
    for (int i = 1; i < kGroup; ++i) most[g] = fmaxf(most[g], x[kGroup * g + i]);
  }
  if ((unsigned)(target - v) < 32u) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (v + i == target) p.z_target[row] = x[i];
  }
  const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  if constexpr (LENGTH > 0) {
    if (__any_sync(0xffffffffu, top > list.above)) {
#pragma unroll
      for (int g = 0; g < 32 / kGroup; ++g)
        if (__any_sync(0xffffffffu, most[g] > list.above)) list.look_through(x + kGroup * g, v + kGroup * g, p.floor + row);
    }
  }
  if constexpr (LENGTH == kKeep) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      stage(list.staging, lane, k, make_uint4(__float_as_uint(x[4 * k]), __float_as_uint(x[4 * k + 1]), __float_as_uint(x[4 * k + 2]),
                                              __float_as_uint(x[4 * k + 3])));
    write_staged(list.rows, list.staging, lane, 4 * (int64_t)v, 4 * p.pitch);
    p.group_top[(int64_t)(v / kRowGroup) * p.n_replicas * p.rows_pad + list.group] = top;
  }
  if (__any_sync(0xffffffffu, top >= s.top && top > -INFINITY)) {
    if (top > s.top) s.raise(top);
    const float m = s.top > -INFINITY ? s.top : NAN;       // equal to nothing
    const float gone = m > -1e37f ? -1e38f : -INFINITY;    // exp of it is 0, and so is 0 times it (-inf: below)
    float n = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const bool is = x[i] == m;
      n += is ? 1.0f : 0.0f;
      x[i] = is ? gone : x[i];
    }
    s.ties += n;
  }
  const float from = s.top > -INFINITY ? s.top : 0.0f;     // nothing finite yet: exp of -inf, not of NaN
  // Two columns an instruction where there is one for it.  The subtraction comes first, as in the loss: in one fma with M log2(e) the rounding of that
  // product is an error of delta that grows with the logits (1e-4 at 2000), and at the ends of the range it is no number.
  const uint64_t scale = pair_of(kLog2e, kLog2e), top2 = pair_of(-from, -from);
  uint64_t e2[2] = {0, 0}, u2[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const uint64_t d = add_pair(pair_of(x[i], x[i + 1]), top2);
    float a, b;
    halves_of(mul_pair(d, scale), a, b);
    const uint64_t y = pair_of(exp2_fast(a), exp2_fast(b));
    e2[i / 2 % 2] = add_pair(e2[i / 2 % 2], y);
    u2[i / 2 % 2] = fma_pair(y, d, u2[i / 2 % 2]);
  }
  float e, u, more;
  halves_of(add_pair(e2[0], e2[1]), e, more);
  e += more;
  halves_of(add_pair(u2[0], u2[1]), u, more);
  u += more;
  if (__any_sync(0xffffffffu, u != u && e == e)) {         // differences of -inf: 0 times them is to be 0, not NaN
    u = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float d = x[i] - from;
      u = fmaf(exp2_fast(d * kLog2e), fmaxf(d, -1e4f), u);
    }
  }
  s.others += e;
  s.weighted += u;
}

// Tiles of (128 * CTAS) x (128 * CTAS) by a resident CTA (or pair): copies, products and readers each go through the same runs, with a ring
// of stages and two accumulators between them.  Every wait is bounded.
//
// The tensor cores cut the sums that they keep instead of rounding them, so a long sum is taken over every kChunk steps: a tile's first
// chunk stays in one accumulator, the next ones go to the other and are added to it by the readers, in fp32 and rounded.  The next tile starts in the
// other one, while the readers go through this tile's sums, 32 columns at a time.  (Sums that were added up in the readers' registers left
// too few for a list: 3.45 ms for 8 x 2048 tokens of width 2048 with 12 entries, against 2.42 without a list.)
// Bound by its readers beside the tensor cores, which are active 60 % of the cycles with 1024 tokens x 50257 of width 1024 and kept logits (99 us), 54 % with
// 8 x 512 tokens and lists (424 us); 8 x 2048 tokens without alternatives take 1.31 ms, 0.83 of the sustained rate of a plain product.
template <int CTAS, int LENGTH>
__global__ void __launch_bounds__(kScoreThreads, 1) scores_kernel(const __grid_constant__ ScoreParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int kTile = 128 * CTAS, kCols = 64 * CTAS;
  const uint32_t smem = (bulk::smem_addr(smem_raw) + 1023u) & ~1023u;
  uint8_t* const behind = smem_raw + (smem - bulk::smem_addr(smem_raw)) + p.stages * kStageBytes;
  Shared& sh = *reinterpret_cast<Shared*>(behind + list_bytes(LENGTH));
  volatile int& failed = sh.failed;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 1 ? 0 : cluster_rank();
  const auto bar = [](const uint64_t& b) { return bulk::smem_addr(&b); };

  let_next_start();
  if (threadIdx.x == 96) {                       // a warp that has nothing else to do
    prefetch_map(&p.weight);
    prefetch_map(&p.hidden);
  }
  if (threadIdx.x == 0) {
    sh.failed = 0;
    for (int s = 0; s < p.stages; ++s) {
      bulk::barrier_init(bar(sh.full[s]), 1);
      bulk::barrier_init(bar(sh.empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      bulk::barrier_init(bar(sh.acc_full[b]), 1);
      bulk::barrier_init(bar(sh.acc_empty[b]), kReaders * CTAS);
    }
    bulk::barrier_init_fence();
  }
  if (warp == 1) tmem_alloc<CTAS>(bulk::smem_addr(&sh.tmem), 2 * 128 * CTAS);
  wait_for_previous();
  if (warp == 2) {
    const int count = lane < p.n_replicas ? p.count[lane] : 0;
    sh.count[lane] = count;
    const int splits = splits_for<CTAS>(p, __reduce_add_sync(0xffffffffu, (count + kTile - 1) / kTile));
    if (lane == 0) {
      sh.splits = splits;
      if (blockIdx.x == 0) p.control->splits = splits;
    }
  }
  fence_before_sync();
  __syncthreads();
  if constexpr (CTAS == 2) cluster_sync();       // the peer's barriers exist before anything arrives there
  fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const int steps = (p.width + kBlockK - 1) / kBlockK, clusters = gridDim.x / CTAS;
  constexpr bool kMajor = false;                 // both operands have the summed axis contiguous
  const auto arrive_leader = [&](uint32_t at) {
    if (rank == 0) bulk::barrier_arrive(at); else arrive_cluster(in_cta(at, 0));
  };

  Run run;
  if (warp == 0) {
    int kb = 0, s = 0;
    uint32_t parity = 0;
    bool go = !p.withhold;
    for (int job = blockIdx.x / CTAS; go && find_run<CTAS>(p, sh, job, run); job += clusters) {
      const int table = p.weight_shared ? 0 : run.r;
      for (int n0 = run.from; go && n0 < run.to; n0 += kTile) {
        const int columns = columns_of<CTAS>(run, n0), boxes = boxes_of<CTAS>(columns);
        const int a_row = run.m0 + 128 * (int)rank, b_row = n0 + columns / CTAS * (int)rank;
        for (int step = 0; step < steps; ++step, ++kb) {
          if (kb >= p.stages && !warp_wait(bar(sh.empty[s]), parity ^ 1, p.wait_limit)) {
            failed = 1;
            go = false;
            break;
          }
          const uint32_t full = bar(sh.full[s]);
          if (rank == 0) expect_bytes(full, CTAS * (kOperandBytes + boxes * kBoxBytes));
          const uint32_t done = CTAS == 1 ? full : in_cta(full, 0);
          const uint32_t dst = smem + s * kStageBytes;
#pragma unroll
          for (int h = 0; h < 2; ++h) load_box<CTAS>(dst + h * kBoxBytes, &p.hidden, step * kBlockK, a_row + 64 * h, run.r, done);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h >= boxes) break;
            load_box<CTAS>(dst + kOperandBytes + h * kBoxBytes, &p.weight, step * kBlockK, b_row + 64 * h, table, done);
          }
          if (++s == p.stages) {
            s = 0;
            parity ^= 1;
          }
        }
        if (__any_sync(0xffffffffu, failed)) go = false;
      }
    }
    // the products have read the last stages: every arrival that was sent to this CTA's barriers is in
    for (int k = kb > p.stages ? kb - p.stages : 0; k < kb && __all_sync(0xffffffffu, !failed); ++k)
      if (!warp_wait(bar(sh.empty[k % p.stages]), (k / p.stages) & 1, p.wait_limit)) failed = 1;
  } else if (warp == 1 && rank == 0) {
    int s = 0, used[2] = {0, 0}, b = 0;
    uint32_t parity = 0;
    bool go = true;
    const uint64_t a_desc = operand_desc(smem, kMajor), b_desc = operand_desc(smem + kOperandBytes, kMajor);
    const uint32_t k_step = k_step_bytes(kMajor);
    for (int job = blockIdx.x / CTAS; go && find_run<CTAS>(p, sh, job, run); job += clusters) {
      for (int n0 = run.from; go && n0 < run.to; n0 += kTile) {
        const uint32_t idesc = instruction_desc<CTAS>(columns_of<CTAS>(run, n0), kMajor, kMajor);
        uint32_t acc = 0;
        for (int step = 0, in_chunk = 0; step < steps; ++step) {
          if (in_chunk == 0) {
            if (step == p.chunk) b ^= 1;         // behind the tile's first chunk
            const int uses = b ? used[1] : used[0];
            if (uses > 0 && !__all_sync(0xffffffffu, wait_cluster(bar(sh.acc_empty[b]), (uses - 1) & 1, 2 * p.wait_limit))) {
              failed = 1;
              go = false;
              break;
            }
            fence_after_sync();
            acc = tmem + b * 128 * CTAS;
          }
          if (!warp_wait(bar(sh.full[s]), parity, p.wait_limit)) {
            failed = 1;
            go = false;
            break;
          }
          fence_after_sync();
#pragma unroll
          for (int k = 0; k < kBlockK / 16; ++k)   // addresses are the descriptors' low bits, in units of 16 bytes
            mma<CTAS>(acc, a_desc + (uint32_t)(s * kStageBytes + k * k_step) / 16, b_desc + (uint32_t)(s * kStageBytes + k * k_step) / 16, idesc,
                      in_chunk > 0 || k > 0);
          commit<CTAS>(bar(sh.empty[s]));
          ++in_chunk;
          if (in_chunk == p.chunk || step + 1 == steps) {
            commit<CTAS>(bar(sh.acc_full[b]));
            if (b) ++used[1]; else ++used[0];
            in_chunk = 0;
          }
          if (++s == p.stages) {
            s = 0;
            parity ^= 1;
          }
        }
        if (steps <= p.chunk) b ^= 1;            // the next tile starts in the accumulator that does not hold this one's sums
        if (__any_sync(0xffffffffu, failed)) go = false;
      }
    }
  } else if (warp >= kFirstReader) {
    const int reader = warp - kFirstReader, quarter = warp & 3, half = reader >> 2;
    const int tile_row = 128 * (int)rank + quarter * 32 + lane, thread = 32 * reader + lane;
    List<LENGTH> list;
    list.at = reinterpret_cast<uint2*>(behind) + thread;
    int used[2] = {0, 0}, b = 0;
    bool go = true;
    const uint32_t my_columns = tmem + half * kCols + ((uint32_t)(quarter * 32) << 16);
    for (int job = blockIdx.x / CTAS; go && find_run<CTAS>(p, sh, job, run); job += clusters) {
      const int64_t row = (int64_t)run.r * p.rows_pad + run.m0 + tile_row;
      const int target = p.target[row];
      State s;
      s.clear();
      if constexpr (LENGTH > 0) {
        list.size = p.list;
        list.clear(__ldcg(p.floor + row));
        if (run.m0 + tile_row >= sh.count[run.r]) list.above = INFINITY;      // zeros behind the counted tokens: nothing is looked for
      }
      if constexpr (LENGTH == kKeep) {
        list.rows.base = reinterpret_cast<char*>(p.logits);
        list.rows.offset = row * p.pitch * 4;
        list.rows.on = __ballot_sync(0xffffffffu, run.m0 + tile_row < sh.count[run.r]);
        list.staging = bulk::smem_addr(behind) + reader * kStagingBytes;
        list.group = row;
      }
      for (int n0 = run.from; go && n0 < run.to; n0 += kTile) {
        const int columns = columns_of<CTAS>(run, n0) - half * kCols;      // that this reader's half has (or none)
        const auto acc_done = [&](int b) {
          fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive_leader(bar(sh.acc_empty[b]));
          if (b) ++used[1]; else ++used[0];
        };
        const auto acc_wait = [&](int b) {
          if (!warp_wait(bar(sh.acc_full[b]), (b ? used[1] : used[0]) & 1, 2 * p.wait_limit)) {
            failed = 1;
            go = false;
          }
          fence_after_sync();
          return go;
        };
        if (!acc_wait(b)) break;
        const uint32_t sums = my_columns + b * 128 * CTAS, chunk = my_columns + (b ^ 1) * 128 * CTAS;
        for (int step = p.chunk; step < steps; step += p.chunk) {
          if (!acc_wait(b ^ 1)) break;
          Columns<CTAS> y;                       // taken at once: the products wait for this accumulator
          take_columns(chunk, y, false);
          acc_done(b ^ 1);
#pragma unroll
          for (int i = 0; i < 4 * CTAS; ++i) {
            float x[16];
            tmem_load16(sums + 16 * i, x);
            tmem_load_wait(x);
#pragma unroll
            for (int k = 0; k < 16; ++k) x[k] += y.x[i / 4][i / 2 % 2][16 * (i % 2) + k];
            tmem_store16(sums + 16 * i, x);
          }
          tmem_store_wait();
        }
        if (!go) break;
#pragma unroll 1
        for (int c = 0; c < min(kCols, columns); c += kColumns) {
          float x[32];
          __syncwarp();
          tmem_load32(sums + c, x);
          tmem_load_wait(x);
          take_logits<LENGTH>(p, x, n0 + half * kCols + c, target, row, s, list);
        }
        acc_done(b);
        b ^= 1;
      }
      if (!go) break;
      const int64_t at = ((int64_t)job * 2 + half) * kTile + tile_row;
      p.part[at] = s;
      if constexpr (LENGTH > 0) {
        list.finish(p.floor + row);
        Key* to = p.lists + ((int64_t)job * 2 + half) * p.list * kTile + tile_row;
        for (int e = 0; e < p.list; ++e) {
          const uint2 u = list.at[e * kReaderThreads];
          const float z = __uint_as_float(u.x);
          to[(int64_t)e * kTile] = z > -INFINITY ? key_of(z, (int)u.y) : 0;
        }
      }
    }
  }
  __syncwarp();
  fence_before_sync();
  __syncthreads();
  if (sh.failed && threadIdx.x == 0) {
    atomicExch(&p.control->status, 1u);
    // copies into this CTA's shared memory and products that read it may still be under way; after this they are not
    for (const long long start = clock64(); clock64() - start < kDrainCycles;) __nanosleep(1000);
  }
  if constexpr (CTAS == 2) cluster_sync();       // neither CTA leaves while the other may still reach into it
  fence_after_sync();
  if (warp == 1) tmem_free<CTAS>(tmem, 2 * 128 * CTAS);
}

// ------------------------------------------------------------------------------------------------ few tokens
// One or two tokens a replica: the table is read once, so that is what bounds it.  A warp takes a run of the table's rows, three at a
// time, a lane 8 elements of each per step.  Every 30 rows (or at the run's end) a lane has one of their logits, and the warp's state and its
// list, sorted, an entry in each lane, take them in together.
// (One token x 50257 of width 768, 12 classes and more: 22.8 us with nothing in the caches, 78 MB from DRAM; 26.5 us for the call.)
constexpr int kFew = 2, kFewRows = 3, kFewBatch = 30;
constexpr int64_t kFewElements = 150000000;      // of all tables, for two tokens: the product is faster beyond

template <int NT>
__global__ void __launch_bounds__(256, 3) few_scores_kernel(const __grid_constant__ ScoreParams p, const __grid_constant__ PackParams k) {
  __shared__ State s_state[8][NT];
  __shared__ Key s_key[8][32];
  let_next_start();
  wait_for_previous();
  const int r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int target[NT], count = 0;
  const __nv_bfloat16* hidden[NT];                 // of the counted tokens, in order
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    target[t] = -1;
    hidden[t] = k.hidden + r * k.hidden_stride;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int y = t < k.n_tokens ? target_of(k, r, t) : -1;
    if (y >= 0) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (i == count) {
          target[i] = k.targets ? y : -1;
          hidden[i] = k.hidden + r * k.hidden_stride + t * k.hidden_row;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && t < k.n_tokens) {
      if (y >= 0) k.token_of[(int64_t)r * p.rows_pad + count] = t;
      else p.out.padding(r, t);
    }
    count += y >= 0;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    k.count[r] = count;
    if (r == 0) p.control->status = 0;
  }
  if (count == 0) return;
  const int64_t w = (int64_t)blockIdx.x * 8 + warp, warps = (int64_t)gridDim.x * 8;
  const int from = (int)(p.vocab * w / warps), to = (int)(p.vocab * (w + 1) / warps);
  const __nv_bfloat16* base = p.table + r * p.table_stride;
  State s[NT];
  Key mine[NT];                                    // this lane's entry of the sorted list
  float held[NT];                                  // this lane's logit of those that wait
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    s[t].clear();
    mine[t] = 0;
    held[t] = -INFINITY;
  }
  int first = from;                                // of those that wait
  const auto take_in = [&](int first) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      s[t].add_warp(held[t]);
      if (p.list) {
        const Key key = held[t] > -INFINITY ? key_of(held[t], first + lane) : 0, last = __shfl_sync(0xffffffffu, mine[t], p.list - 1);
        if (__any_sync(0xffffffffu, key > last)) mine[t] = merged(mine[t], sorted(key));
      }
      held[t] = -INFINITY;
    }
  };
  for (int v = from; v < to; v += kFewRows) {
    float z[kFewRows][NT];
    const __nv_bfloat16* row[kFewRows];
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      row[i] = base + min(v + i, to - 1) * p.table_row;   // behind the run's end: its last row again, not counted
#pragma unroll
      for (int t = 0; t < NT; ++t) z[i][t] = 0.0f;
    }
#pragma unroll 3
    for (int c = lane * 8; c < p.width; c += 256) {
      uint4 u[kFewRows];
#pragma unroll
      for (int i = 0; i < kFewRows; ++i) u[i] = __ldcs(reinterpret_cast<const uint4*>(row[i] + c));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint4 h4 = *reinterpret_cast<const uint4*>(hidden[t] + c);
        const uint32_t h[4] = {h4.x, h4.y, h4.z, h4.w};
#pragma unroll
        for (int i = 0; i < kFewRows; ++i) {
          const uint32_t x[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            z[i][t] = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(h[e] << 16), z[i][t]);
            z[i][t] = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(h[e] & 0xffff0000u), z[i][t]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kFewRows; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z[i][t] += __shfl_xor_sync(0xffffffffu, z[i][t], o);
        if (v + i >= to) continue;
        if (v + i - first == lane) held[t] = z[i][t];
        if (v + i == target[t] && lane == 0) p.z_target[(int64_t)r * p.rows_pad + t] = z[i][t];
      }
    if (v + kFewRows - first == kFewBatch || v + kFewRows >= to) {
      take_in(first);
      first = v + kFewRows;
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
    if (lane == 0) s_state[warp][t] = s[t];
  __syncthreads();
  if (threadIdx.x < count) {
    State all = s_state[0][threadIdx.x];
    for (int i = 1; i < 8; ++i) all.add(s_state[i][threadIdx.x]);
    p.part[((int64_t)r * kFew + threadIdx.x) * p.n_parts + blockIdx.x] = all;
  }
  if (!p.list) return;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t >= count) break;
    const Key key = merged_of_warps<8>(mine[t], warp, s_key);
    if (warp == 0 && lane < p.list) p.lists[(((int64_t)r * kFew + t) * p.n_parts + blockIdx.x) * p.list + lane] = key;
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ joining
__host__ __device__ constexpr int join_rows(int warps) { return warps == 1 ? 8 : 1; }        // rows a block
__host__ __device__ constexpr int join_threads(int warps) { return 32 * warps * join_rows(warps); }
constexpr int kMostCands = 256;                    // candidates of a row; more of them take a longer way

// WARPS warps a row: all of a block where rows are few, one where they are many.  The row's lists (or, KEPT, its groups of 32 logits) hold
// its C best.  Any C of their entries give a bound that the C best are not below: the C-th of the lists' first entries (of the threads' best
// of them), or, with few lists, of their first entries, second ones, and so on.  The entries at or above it are hardly more than C; they are
// collected and sorted.
// The C classes' logits are then formed again in fp64, which decides their order; a row gathers C rows of the table for it, mostly from L2,
// and that is what bounds the kernel (8 x 512 tokens of width 1024, 12 classes: 50 us; 1024 tokens of kept logits 44 us).
template <int CTAS, int WARPS, bool KEPT = false>  // CTAS 0: after few_scores_kernel
__global__ void __launch_bounds__(join_threads(WARPS)) join_scores_kernel(const __grid_constant__ ScoreParams p) {
  constexpr int kTile = CTAS ? 128 * CTAS : 1, kRows = join_rows(WARPS), kRowThreads = 32 * WARPS;
  __shared__ float s_state[WARPS][4], s_head[WARPS][32];
  __shared__ Key s_key[WARPS][32], s_best[kRows][32], s_cand[kRows][kMostCands];
  __shared__ int s_list[kRows][kMostCands], s_lists[kRows], s_cands[kRows];
  __shared__ long long s_exact[kRows][32];         // doubles as integers of the same order
  const int lane = threadIdx.x & 31, in_block = (threadIdx.x >> 5) / WARPS, warp = (threadIdx.x >> 5) % WARPS, thread = 32 * warp + lane;
  const int r = blockIdx.y, row = blockIdx.x * kRows + in_block;
  const auto sync = [] { if constexpr (WARPS == 1) __syncwarp(); else __syncthreads(); };
  let_next_start();
  if (thread == 0) s_lists[in_block] = s_cands[in_block] = 0;
  wait_for_previous();
  const int64_t at = (int64_t)r * p.rows_pad + row;
  const int count = p.count[r], splits = CTAS ? p.control->splits : 0;
  const unsigned status = CTAS ? p.control->status : 0;
  if (row >= count) return;                        // (all of a row's warps)
  const int token = p.token_of[at];
  const float z_target = p.out.logprob.p ? p.z_target[at] : 0.0f;
  // where this row's states and lists are
  int parts = p.n_parts, row_tiles = 0;
  int64_t first_job = 0;
  if constexpr (CTAS) {
    for (int i = 0; i < r; ++i) first_job += (p.count[i] + kTile - 1) / kTile;
    first_job = first_job * splits + row / kTile;
    row_tiles = (count + kTile - 1) / kTile;
    parts = 2 * splits;
  }
  const auto part_at = [&](int l) -> int64_t {
    if constexpr (CTAS) return ((first_job + (int64_t)(l >> 1) * row_tiles) * 2 + (l & 1)) * kTile + row % kTile;
    else return ((int64_t)r * kFew + row) * p.n_parts + l;
  };
  const auto entry = [&](int l, int e) -> Key {
    if constexpr (KEPT) {
      const float z = p.logits[at * p.pitch + l * kRowGroup + e];
      return z > -INFINITY ? key_of(z, l * kRowGroup + e) : 0;
    } else if constexpr (CTAS) {
      return p.lists[(((first_job + (int64_t)(l >> 1) * row_tiles) * 2 + (l & 1)) * p.list + e) * kTile + row % kTile];
    } else {
      return p.lists[part_at(l) * p.list + e];
    }
  };
  const auto logit = [](Key key) { return key ? logit_of(key) : -INFINITY; };
  const auto first_of = [&](int l) -> float {      // the largest of the list's logits
    if constexpr (KEPT) return p.group_top[(int64_t)l * p.n_replicas * p.rows_pad + at];
    else return logit(entry(l, 0));
  };
  // the lists' largest logits, under way with the states
  const int list = p.list, n_top = p.out.n_top;
  const int lists = KEPT ? (p.vocab + kRowGroup - 1) / kRowGroup : parts, entries = KEPT ? kRowGroup : list;
  constexpr int kHeads = 4;                        // lists a thread whose largest logits stay in registers
  float heads[kHeads], head = -INFINITY;
  const bool flat = !KEPT && lists * entries <= 8 * kRowThreads;       // few enough to look at all entries
  if (flat) {
    if (p.list && thread < lists * entries) head = logit(entry(thread % lists, thread / lists));
  } else if (p.list) {
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
      heads[k] = thread + k * kRowThreads < lists ? first_of(thread + k * kRowThreads) : -INFINITY;
      head = fmaxf(head, heads[k]);
    }
#pragma unroll 4
    for (int l = thread + kHeads * kRowThreads; l < lists; l += kRowThreads) head = fmaxf(head, first_of(l));
  }
  State s;
  s.clear();
  for (int l = thread; l < parts; l += kRowThreads) s.add(p.part[part_at(l)]);
  s.add_all<WARPS>(warp, s_state);
  // the logarithm of the sum less the maximum's: >= 0
  float rest = logf(s.ties) + log1pf(s.others / s.ties);
  if (status != 0 || !(fabsf(s.top) < INFINITY) || !(rest < INFINITY)) rest = NAN;
  const ScoreOut& o = p.out;
  if (thread == 0) {
    if (o.lse.p) o.lse.at(r, token) = s.top + rest;
    if (o.entropy.p) o.entropy.at(r, token) = rest - s.weighted / (s.ties + s.others);
    if (o.logprob.p) o.logprob.at(r, token) = -((s.top - z_target) + rest);
  }
  if (!list) return;
  const int64_t out_at = (int64_t)token * n_top;
  if (rest != rest) {
    if (thread < n_top) {
      o.top_ids.at(r, out_at + thread) = -1;
      if (o.top_logprob.p) o.top_logprob.at(r, out_at + thread) = NAN;
    }
    return;
  }
  // the bound
  head = sorted(head);
  if constexpr (WARPS > 1) {
    head = merged_of_warps<WARPS>(head, warp, s_head);
    if (warp == 0) s_head[0][lane] = head;
    __syncthreads();
    head = s_head[0][list - 1];
  } else {
    head = __shfl_sync(0xffffffffu, head, list - 1);
    __syncwarp();                                  // the counters are zero
  }
  const Key bound = head > -INFINITY ? key_of(head, -1) : 1;      // of all ids; 1: fewer than C
  // what is not below it
  const unsigned before_me = (1u << lane) - 1;
  int found = 0, cands = 0;                        // of a warp that is alone with its row
  const auto place_of = [&](bool is, int& mine, int* shared) {       // in a list of the row's; of a warp's threads together
    const unsigned some = __ballot_sync(0xffffffffu, is);
    int first = mine;
    if constexpr (WARPS == 1) {
      mine += __popc(some);
    } else if (some) {
      if (lane == 0) first = atomicAdd(shared, __popc(some));
      first = __shfl_sync(0xffffffffu, first, 0);
    }
    return first + __popc(some & before_me);
  };
  const auto collect = [&](Key key) {
    const int place = place_of(key >= bound, cands, &s_cands[in_block]);
    if (key >= bound && place < kMostCands) s_cand[in_block][place] = key;
  };
  bool all = true;
  if (flat) {
#pragma unroll 4
    for (int c = thread - lane; c < lists * entries; c += kRowThreads)
      collect(c + lane < lists * entries ? entry((c + lane) % lists, (c + lane) / lists) : 0);
  } else {
    const auto look = [&](int l, float largest) {
      const bool is = l < lists && largest >= head;
      const int place = place_of(is, found, &s_lists[in_block]);
      if (is && place < kMostCands) s_list[in_block][place] = l;
    };
#pragma unroll
    for (int k = 0; k < kHeads; ++k) look(thread + k * kRowThreads, heads[k]);
    for (int l = thread - lane + kHeads * kRowThreads; l < lists; l += kRowThreads) look(l + lane, l + lane < lists ? first_of(l + lane) : -INFINITY);
    sync();
    if constexpr (WARPS > 1) found = s_lists[in_block];
    all = found <= kMostCands;
    constexpr int kListsAtOnce = WARPS == 1 ? 8 : 2;
    for (int i = warp; i < min(found, kMostCands); i += kListsAtOnce * WARPS) {
      Key key[kListsAtOnce];
#pragma unroll
      for (int k = 0; k < kListsAtOnce; ++k)
        key[k] = i + k * WARPS < min(found, kMostCands) && lane < entries ? entry(s_list[in_block][i + k * WARPS], lane) : 0;
#pragma unroll
      for (int k = 0; k < kListsAtOnce; ++k) collect(key[k]);
    }
  }
  sync();
  if constexpr (WARPS > 1) cands = s_cands[in_block];
  Key mine = 0;
  const bool collected = all && cands <= kMostCands;
  if (collected) {
    for (int c = 32 * warp; c < cands; c += kRowThreads) {
      const Key key = sorted(c + lane < cands ? s_cand[in_block][c + lane] : 0);
      mine = mine ? merged(mine, key) : key;
    }
  } else {                                         // many equal or nearly equal logits: every list after the other
    for (int l = warp; l < lists; l += WARPS) {
      const Key key = lane < entries ? entry(l, lane) : 0, last = __shfl_sync(0xffffffffu, mine, list - 1);
      if (__any_sync(0xffffffffu, key > last)) mine = merged(mine, sorted(key));
    }
  }
  if (WARPS > 1 && (!collected || cands > 32)) mine = merged_of_warps<WARPS>(mine, warp, s_key);
  if (warp == 0) s_best[in_block][lane] = mine;
  sync();
  // their logits in fp64, kAtOnce classes and kAhead x 256 columns of them at a time, all loads before the first sum
  const __nv_bfloat16* h = p.rows + r * p.rows_stride + (p.rows_packed ? row : token) * p.rows_row;
  const __nv_bfloat16* table = p.table + (p.weight_shared ? 0 : r * p.table_stride);
  constexpr int kAtOnce = WARPS >= 32 ? 1 : WARPS > 1 ? 2 : 4, kAhead = 3;
  for (int e0 = warp; e0 < list; e0 += kAtOnce * WARPS) {
    const __nv_bfloat16* w[kAtOnce];
    double sum[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const Key key = e0 + i * WARPS < list ? s_best[in_block][e0 + i * WARPS] : 0;
      w[i] = table + (key ? class_of(key) : 0) * p.table_row;
      sum[i] = 0.0;
    }
    const int whole = p.rows_vec ? p.width & ~7 : 0;
    for (int c0 = lane * 8; c0 < whole; c0 += 256 * kAhead) {
      uint4 a4[kAhead], b4[kAtOnce][kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        const int c = c0 + 256 * q;
        if (c >= whole) continue;
        a4[q] = *reinterpret_cast<const uint4*>(h + c);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (e0 + i * WARPS < list) b4[i][q] = *reinterpret_cast<const uint4*>(w[i] + c);
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (c0 + 256 * q >= whole) continue;
        const uint32_t a[4] = {a4[q].x, a4[q].y, a4[q].z, a4[q].w};
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          if (e0 + i * WARPS >= list) continue;
          const uint32_t b[4] = {b4[i][q].x, b4[i][q].y, b4[i][q].z, b4[i][q].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {            // a product of two bf16 numbers is an fp32 number
            sum[i] += (double)(__uint_as_float(a[k] << 16) * __uint_as_float(b[k] << 16));
            sum[i] += (double)(__uint_as_float(a[k] & 0xffff0000u) * __uint_as_float(b[k] & 0xffff0000u));
          }
        }
      }
    }
    for (int c = whole + lane; c < p.width; c += 32)
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) sum[i] += (double)(__bfloat162float(h[c]) * __bfloat162float(w[i][c]));
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
#pragma unroll
      for (int k = 16; k > 0; k >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], k);
      const long long u = __double_as_longlong(sum[i] + 0.0);
      if (lane == 0 && e0 + i * WARPS < list) s_exact[in_block][e0 + i * WARPS] = u < 0 ? u ^ 0x7fffffffffffffffll : u;
    }
  }
  sync();
  if (warp != 0 || lane >= list) return;
  const Key key = s_best[in_block][lane];
  int place = lane;                                // of an entry that holds nothing
  if (key) {
    const long long z = s_exact[in_block][lane];
    const int id = class_of(key);
    place = 0;
#pragma unroll 8
    for (int i = 0; i < list; ++i) {
      const Key other = s_best[in_block][i];
      const long long y = s_exact[in_block][i];
      place += (other != 0) & ((y > z) | ((y == z) & (class_of(other) < id)));      // (no branch, so that the loads go on)
    }
  }
  if (place < n_top) {
    o.top_ids.at(r, out_at + place) = key ? class_of(key) : -1;
    if (o.top_logprob.p) o.top_logprob.at(r, out_at + place) = key ? -((s.top - logit_of(key)) + rest) : -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------------ host side
constexpr int kSms = 148;        // of a B200, for sizes that must not depend on the device; with another count only times change
// Rows that are joined by a block of 32 warps each (two rounds of them at most), and from where on a warp alone takes one; 8 warps between.
// (3 x 777 tokens of a vocabulary of 4099, width 520: 56 us for the call with a warp a row, 70 with 8.)
constexpr int64_t kFewRowsToJoin = 2 * kSms, kManyRows = 2048;
// Logits that are kept for the join to look through, in place of lists that are held while they are formed: writing and reading them is 8 bytes
// each, lists cost a start and the merges of a run, which are dear where runs are short.  (1024 tokens x 50257 of width 1024, 51 M logits: 146 us
// kept and 173 with lists for 8 alternatives, 165 and 273 for 20; 2048 tokens, 103 M: 260 and 245 for 8, 274 and 266 for 12, but 284 and 346 for 13, 310 and 398
// for 20: for more than 12 alternatives, whose lists are longer, this is too low; 8 x 2048 tokens, 823 M: 2095 and 1450 for 8, 2218 and 1867 for 20.)
constexpr int64_t kKeepLogits = 64ll << 20;      // 256 MB

// Whether the table's boxes can be copied from where it is.
bool table_fits(const hdet_token_scores_args* d) {
  return aligned(d->weight, 16) && d->weight_row % 8 == 0 && (d->n_replicas == 1 || d->weight_stride % 8 == 0);
}

constexpr int64_t kFewBlocks = kSms * 3;        // blocks of few_scores_kernel that are resident at once

struct Plan {
  int ctas, tile, list, held;
  int64_t rows_pad, packed_row, m_tiles, n_tiles;
  bool few, pack_table;
  int64_t n_parts;                // of few_scores_kernel
  int64_t most_jobs, pitch;
  int64_t off_count, off_target, off_token, off_z, off_floor, off_part, off_lists, off_logits, off_groups, off_hidden, off_table, total;
};

Plan plan_of(const hdet_token_scores_args* d) {
  Plan q{};
  const int64_t R = d->n_replicas, T = d->n_tokens, V = d->vocab, D = d->width;
  // as in the loss: pairs share operands, single CTAs make four times as many tiles
  q.ctas = T <= 192 || R * div_up(T, 256) * div_up(V, 256) < 64 ? 1 : 2;
  q.tile = 128 * q.ctas;
  q.rows_pad = round_up(T > 0 ? T : 1, q.tile);
  q.packed_row = round_up(D, 8);
  q.m_tiles = q.rows_pad / q.tile;
  q.n_tiles = div_up(V, q.tile);
  q.list = d->n_top ? (int)std::min<int64_t>(d->n_top + kMargin, V) : 0;
  q.pitch = q.n_tiles * q.tile;
  q.held = !q.list ? kNoList : R * q.rows_pad * q.pitch <= kKeepLogits ? kKeep : q.list <= kShort ? kShort : kLong;
  q.pack_table = !table_fits(d);
  q.few = T > 0 && T <= kFew && (T == 1 || R * V * D <= kFewElements) && !q.pack_table && D % 8 == 0 && aligned(d->hidden, 16) &&
          d->hidden_row % 8 == 0 && (R == 1 || d->hidden_stride % 8 == 0);
  const int64_t most = div_up(V, 8 * kFewRows), blocks = std::max<int64_t>(1, kFewBlocks / R);
  q.n_parts = std::min(blocks, most);
  // Four rounds of jobs are enough to even out their ends; a row has a state and a list from each run and half.
  const int64_t row_tiles = R * q.m_tiles;
  q.most_jobs = std::max<int64_t>(row_tiles, 4 * kSms / q.ctas);
  int64_t at = round_up(sizeof(Control), 256);
  const auto take = [&](int64_t bytes) { const int64_t o = at; at = round_up(at + bytes, 256); return o; };
  q.off_count = take(4 * R);
  q.off_target = take(4 * R * q.rows_pad);
  q.off_token = take(4 * R * q.rows_pad);
  q.off_z = take(4 * R * q.rows_pad);
  q.off_floor = take(4 * R * q.rows_pad);
  // room for either kernel's: which one runs depends on the hidden states' address, and the size does not
  const int64_t states = std::max<int64_t>(q.most_jobs * 2 * q.tile, T <= kFew ? R * kFew * q.n_parts : 0);
  q.off_part = take(16 * states);
  q.off_lists = take(q.held > 0 || T <= kFew ? 8 * states * q.list : 0);
  if (q.held == kKeep) {
    q.off_logits = take(4 * R * q.rows_pad * q.pitch);
    q.off_groups = take(4 * R * q.rows_pad * (q.pitch / kRowGroup));
  }
  q.off_hidden = take(2 * R * q.rows_pad * q.packed_row);
  if (q.pack_table) q.off_table = take(2 * (R > 1 && d->weight_stride ? R : 1) * V * q.packed_row);
  q.total = at;
  return q;
}

// The most that a call with up to n_tokens tokens needs: with more tokens everything but the number of jobs grows, and that is the
// same below four rounds of them; only the two tile sizes differ.
int64_t workspace_of(const hdet_token_scores_args* d) {
  hdet_token_scores_args a = *d;
  int64_t most = plan_of(d).total;
  for (a.n_tokens = kFew; a.n_tokens < d->n_tokens; a.n_tokens = a.n_tokens == kFew ? 64 : a.n_tokens + 64)
    most = std::max(most, plan_of(&a).total);
  return most;
}

template <int CTAS>
auto pick_kernel(int held) {
  return held == kNoList ? scores_kernel<CTAS, kNoList> : held == kKeep ? scores_kernel<CTAS, kKeep> : held == kShort ? scores_kernel<CTAS, kShort> : scores_kernel<CTAS, kLong>;
}

cudaError_t prepare(int device, int* sms) {
  const void* kernels[] = {
#define HDET_LENGTHS(ctas)                                                                             \
  (const void*)scores_kernel<ctas, kNoList>, (const void*)scores_kernel<ctas, kKeep>,                  \
      (const void*)scores_kernel<ctas, kShort>, (const void*)scores_kernel<ctas, kLong>
      HDET_LENGTHS(1), HDET_LENGTHS(2)};
#undef HDET_LENGTHS
  return prepare_device(device, sms, kernels, kMaxSmem);
}

}  // namespace

int check_token_scores(const char* who, const hdet_token_scores_args* d, bool gradient) {
  if (!d) return fail(HDET_ERR_INVALID_ARG, who, "the descriptor is NULL");
  if (d->n_replicas < 1 || d->n_replicas > HDET_MAX_REPLICAS)
    return fail(HDET_ERR_INVALID_ARG, who, "n_replicas must be in 1..32");
  if (d->n_tokens < 0 || d->n_tokens > HDET_MAX_TOKENS || d->vocab < 1 || d->vocab > HDET_MAX_VOCAB || d->width < 1 ||
      d->width > HDET_MAX_WIDTH)
    return fail(HDET_ERR_INVALID_ARG, who, "n_tokens, vocab or width out of range");
  if (!gradient && (d->n_top < 0 || d->n_top > HDET_MAX_TOP || d->n_top > d->vocab))
    return fail(HDET_ERR_INVALID_ARG, who, "n_top must be in 0..20 and at most vocab");
  if (d->target_dtype != HDET_DTYPE_I32 && d->target_dtype != HDET_DTYPE_I64)
    return fail(HDET_ERR_INVALID_ARG, who, "target_dtype must be HDET_DTYPE_I32 or HDET_DTYPE_I64");
  if (d->hidden_dtype != HDET_DTYPE_BF16 || d->weight_dtype != HDET_DTYPE_BF16) {
    if (!is_float(d->hidden_dtype) || !is_float(d->weight_dtype))
      return fail(HDET_ERR_INVALID_ARG, who, "hidden_dtype and weight_dtype must be HDET_DTYPE_*");
    return fail(HDET_ERR_UNSUPPORTED, who, "hidden states and table must be HDET_DTYPE_BF16 (hdet_tensor.param_bf16, or a bf16 copy)");
  }
  if (d->device < 0) return fail(HDET_ERR_INVALID_ARG, who, "device must be >= 0");
  if (d->hidden_row < d->width || d->weight_row < d->width) return fail(HDET_ERR_INVALID_ARG, who, "a row stride is smaller than width");
  if (std::max(d->hidden_row, d->weight_row) > HDET_MAX_ROW_STRIDE) return fail(HDET_ERR_INVALID_ARG, who, "a row stride is out of range");
  if (gradient) {
    if ((d->d_hidden && !is_float(d->d_hidden_dtype)) || (d->d_weight && !is_float(d->d_weight_dtype)))
      return fail(HDET_ERR_INVALID_ARG, who, "the gradients' dtypes must be HDET_DTYPE_F32 or HDET_DTYPE_BF16");
    if (d->piece_bytes < 0) return fail(HDET_ERR_INVALID_ARG, who, "piece_bytes must be >= 0");
    if ((d->d_hidden && d->d_hidden_row < d->width) || (d->d_weight && d->d_weight_row < d->width))
      return fail(HDET_ERR_INVALID_ARG, who, "a row stride is smaller than width");
    if ((d->d_hidden && d->d_hidden_row > HDET_MAX_ROW_STRIDE) || (d->d_weight && d->d_weight_row > HDET_MAX_ROW_STRIDE))
      return fail(HDET_ERR_INVALID_ARG, who, "a row stride is out of range");
  }
  if (d->n_replicas == 1) return HDET_OK;
  const int64_t strides[] = {d->hidden_stride,   d->weight_stride,      d->target_stride,    d->logprob_stride,   d->entropy_stride,  d->lse_stride,
                             d->top_ids_stride, d->top_logprob_stride, d->d_logprob_stride, d->d_entropy_stride, d->d_hidden_stride, d->d_weight_stride};
  for (const int64_t s : strides) {
    if (s < 0) return fail(HDET_ERR_INVALID_ARG, who, "negative stride");
    if (s > HDET_MAX_REPLICA_STRIDE) return fail(HDET_ERR_INVALID_ARG, who, "a replica stride is out of range");
  }
  return HDET_OK;
}

int check_token_scores_pointers(const char* who, const hdet_token_scores_args* d, bool gradient) {
  const int64_t T = d->n_tokens;
  if (!d->weight || (T > 0 && !d->hidden)) return fail(HDET_ERR_INVALID_ARG, who, "a pointer is NULL");
  const auto span = [&](int64_t rows, int64_t row) { return rows > 0 ? (rows - 1) * row + d->width : 0; };
  struct PerTokenArray { const void* p; int64_t stride, each; };
  const PerTokenArray scores[] = {{d->logprob, d->logprob_stride, 1}, {d->entropy, d->entropy_stride, 1}, {d->lse, d->lse_stride, 1}};
  const PerTokenArray out[] = {{d->top_ids, d->top_ids_stride, d->n_top}, {d->top_logprob, d->top_logprob_stride, d->n_top}};
  const PerTokenArray given[] = {{d->d_logprob, d->d_logprob_stride, 1}, {d->d_entropy, d->d_entropy_stride, 1}};
  const bool many = d->n_replicas > 1;
  // written arrays have a replica's values apart; what a gradient reads may be one array for all
  const auto fits = [&](const PerTokenArray& a, bool read) { return !many || !a.p || a.stride >= T * a.each || (read && a.stride == 0); };
  bool strides = true, alignment = aligned(d->hidden, 2) && aligned(d->weight, 2) && aligned(d->targets, d->target_dtype == HDET_DTYPE_I64 ? 8 : 4);
  for (const auto& a : scores) {
    strides = strides && fits(a, gradient);
    alignment = alignment && aligned(a.p, 4);
  }
  if (gradient) {
    if (!d->d_hidden && !d->d_weight) return fail(HDET_ERR_INVALID_ARG, who, "no gradient is asked for");
    if (T > 0 && !d->d_logprob && !d->d_entropy) return fail(HDET_ERR_INVALID_ARG, who, "d_logprob and d_entropy are both NULL");
    if (T > 0 && (!d->lse || (d->targets && !d->logprob) || (d->d_entropy && !d->entropy)))
      return fail(HDET_ERR_INVALID_ARG, who, "lse, logprob (with targets) and entropy (with d_entropy) must be given");
    if (T > 0 && d->d_logprob && !d->targets) return fail(HDET_ERR_INVALID_ARG, who, "d_logprob needs targets");
    for (const auto& a : given) {
      strides = strides && fits(a, true);
      alignment = alignment && aligned(a.p, 4);
    }
    if (many && ((d->d_hidden && d->d_hidden_stride < span(T, d->d_hidden_row)) || (d->d_weight && d->d_weight_stride < span(d->vocab, d->d_weight_row))))
      strides = false;
    alignment = alignment && (!d->d_hidden || aligned(d->d_hidden, elem_size(d->d_hidden_dtype))) &&
                (!d->d_weight || aligned(d->d_weight, elem_size(d->d_weight_dtype)));
    // In the hidden states' own buffer every row of d_hidden has to lie on its own hidden state's: other rows are still to be read.
    if (d->d_hidden && d->d_hidden == d->hidden && T > 0 &&
        (d->d_hidden_dtype != HDET_DTYPE_BF16 || d->d_hidden_row != d->hidden_row || (many && d->d_hidden_stride != d->hidden_stride)))
      return fail(HDET_ERR_INVALID_ARG, who, "d_hidden in the place of the hidden states needs their dtype and strides");
  } else {
    if (T > 0 && !d->logprob && !d->entropy && !d->lse && !d->n_top) return fail(HDET_ERR_INVALID_ARG, who, "no output is asked for");
    if (T > 0 && d->logprob && !d->targets) return fail(HDET_ERR_INVALID_ARG, who, "logprob needs targets");
    if (T > 0 && ((d->n_top > 0) != (d->top_ids != nullptr) || (d->top_logprob && !d->top_ids)))
      return fail(HDET_ERR_INVALID_ARG, who, "top_ids goes with n_top, and top_logprob with both");
    for (const auto& a : out) {
      strides = strides && fits(a, false);
      alignment = alignment && aligned(a.p, 4);
    }
  }
  if (many && ((d->hidden_stride && d->hidden_stride < span(T, d->hidden_row)) || (d->weight_stride && d->weight_stride < span(d->vocab, d->weight_row)) ||
               (d->targets && d->target_stride && d->target_stride < T)))
    strides = false;
  if (!strides) return fail(HDET_ERR_INVALID_ARG, who, "a replica stride is smaller than one replica");
  if (!alignment) return fail(HDET_ERR_ALIGN, who, "a pointer is not aligned to its element type");
  return HDET_OK;
}

namespace {

template <typename T>
PerToken<T> per_token(void* p, int64_t stride, bool many) { return PerToken<T>{static_cast<T*>(p), many ? stride : 0}; }

int token_scores(const char* who, const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream, bool selftest) {
  TraceRange trace(who);
  if (const int rc = check_token_scores(who, d, false)) return rc;
  if (const int rc = check_token_scores_pointers(who, d, false)) return rc;
  const Plan q = plan_of(d);
  if (!workspace || workspace_bytes < q.total)
    return fail(HDET_ERR_INVALID_ARG, who, "the workspace is NULL or smaller than hdet_token_scores_workspace says");
  if (!aligned(workspace, 256)) return fail(HDET_ERR_ALIGN, who, "the workspace is not 256-byte aligned");
  if (q.m_tiles * q.n_tiles * d->n_replicas * q.ctas > INT32_MAX || q.rows_pad * q.packed_row * 2 >= (1ll << 40) ||
      d->weight_row * d->vocab * 2 >= (1ll << 40) || (d->n_replicas > 1 && d->weight_stride * 2 >= (1ll << 40)))
    return fail(HDET_ERR_UNSUPPORTED, who, "too many tiles, or a stride of 2^40 bytes or more");
  if (selftest && q.few) return fail(HDET_ERR_UNSUPPORTED, who, "the kernel for so few tokens waits for nothing");
  if (d->n_tokens == 0) return HDET_OK;
  DeviceScope scope(d->device);
  if (scope.err != cudaSuccess) return fail_cuda(who, scope.err);
  int sms = 0;
  cudaError_t e = prepare(d->device, &sms);
  if (e != cudaSuccess) return fail_cuda(who, e);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const bool many = d->n_replicas > 1;
  const bool shared_table = !many || d->weight_stride == 0;

  ScoreParams p{};
  p.n_replicas = d->n_replicas;
  p.vocab = (int)d->vocab; p.width = (int)d->width; p.n_tokens = (int)d->n_tokens; p.rows_pad = (int)q.rows_pad;
  p.weight_shared = shared_table;
  p.count = reinterpret_cast<int*>(ws + q.off_count);
  p.target = reinterpret_cast<int*>(ws + q.off_target);
  p.token_of = reinterpret_cast<int*>(ws + q.off_token);
  p.z_target = reinterpret_cast<float*>(ws + q.off_z);
  p.part = reinterpret_cast<State*>(ws + q.off_part);
  p.floor = reinterpret_cast<int*>(ws + q.off_floor);
  p.lists = reinterpret_cast<Key*>(ws + q.off_lists);
  p.n_parts = (int)q.n_parts;
  p.n_units = (int)div_up(d->vocab, unit_of(q.ctas));
  p.list = q.list;
  p.most_jobs = (int)std::min<int64_t>(q.most_jobs, INT32_MAX);
  p.chunk = kChunk;
  p.control = reinterpret_cast<Control*>(ws);
  p.wait_limit = selftest ? kSelftestLimitCycles : bulk::kWaitLimitCycles;
  p.withhold = selftest;
  p.out.logprob = per_token<float>(d->logprob, d->logprob_stride, many);
  p.out.entropy = per_token<float>(d->entropy, d->entropy_stride, many);
  p.out.lse = per_token<float>(d->lse, d->lse_stride, many);
  p.out.top_logprob = per_token<float>(d->top_logprob, d->top_logprob_stride, many);
  p.out.top_ids = per_token<int>(d->top_ids, d->top_ids_stride, many);
  p.out.n_top = d->n_top;
  p.logits = reinterpret_cast<float*>(ws + q.off_logits);
  p.group_top = reinterpret_cast<float*>(ws + q.off_groups);
  p.pitch = q.pitch;
  p.out.floor = q.held > 0 && !q.few ? p.floor : nullptr;

  PackParams k{};
  k.hidden = static_cast<const __nv_bfloat16*>(d->hidden);
  k.hidden_stride = many ? d->hidden_stride : 0;
  k.hidden_row = d->hidden_row;
  k.targets = d->targets;
  k.target_stride = many ? d->target_stride : 0;
  k.wide = d->target_dtype == HDET_DTYPE_I64;
  k.hidden_vec = aligned(d->hidden, 16) && d->hidden_row % 8 == 0 && k.hidden_stride % 8 == 0 && d->width % 8 == 0;
  k.n_tokens = p.n_tokens; k.vocab = p.vocab; k.width = p.width; k.rows_pad = p.rows_pad; k.row_tile = q.tile;
  k.packed_row = (int)q.packed_row;
  k.packed = reinterpret_cast<__nv_bfloat16*>(ws + q.off_hidden);
  k.count = const_cast<int*>(p.count);
  k.target = const_cast<int*>(p.target);
  k.token_of = const_cast<int*>(p.token_of);
  k.control = p.control;
  p.table = static_cast<const __nv_bfloat16*>(d->weight);
  p.table_row = d->weight_row;
  p.table_stride = shared_table ? 0 : d->weight_stride;
  const int tables = shared_table ? 1 : d->n_replicas;
  const auto join = [&](auto kernel, int warps) {
    return launch(kernel, dim3((unsigned)div_up(d->n_tokens, join_rows(warps)), d->n_replicas), join_threads(warps), 0, 1, st, p);
  };
  if (q.few) {
    p.rows = k.hidden; p.rows_stride = k.hidden_stride; p.rows_row = k.hidden_row;
    p.rows_vec = true;
    const dim3 grid((unsigned)q.n_parts, d->n_replicas);
    e = launch(d->n_tokens == 1 ? few_scores_kernel<1> : few_scores_kernel<2>, grid, 256, 0, 1, st, p, k);
    if (e == cudaSuccess) e = join(join_scores_kernel<0, 16>, 16);
    return e == cudaSuccess ? HDET_OK : fail_cuda(who, e);
  }
  const int64_t pack_rows = round_up(div_up(d->n_tokens, kPackBlocks), 8);
  e = launch(pack_kernel<kPackScores, ScoreOut>, dim3((unsigned)div_up(d->n_tokens, pack_rows), d->n_replicas), 256, 0, 1, st, k, (int)pack_rows, p.out);
  if (e != cudaSuccess) return fail_cuda(who, e);
  if (q.pack_table) {
    __nv_bfloat16* packed = reinterpret_cast<__nv_bfloat16*>(ws + q.off_table);
    e = launch_pack_table(p.table, shared_table ? 0 : d->weight_stride, d->weight_row, p.vocab, p.width, k.packed_row, tables, packed, st);
    if (e != cudaSuccess) return fail_cuda(who, e);
    p.table = packed;
    p.table_row = q.packed_row;
    p.table_stride = q.packed_row * d->vocab;
  }
  p.rows = k.packed; p.rows_stride = q.rows_pad * q.packed_row; p.rows_row = q.packed_row;
  p.rows_packed = p.rows_vec = true;
  if (!encode(&p.hidden, k.packed, d->width, q.rows_pad, d->n_replicas, q.packed_row, q.rows_pad * q.packed_row) ||
      !encode(&p.weight, p.table, d->width, d->vocab, tables, p.table_row, shared_table ? p.table_row * d->vocab : p.table_stride))
    return fail(HDET_ERR_CUDA, who, "the driver refused a tensor map");
  // every cluster that finds a job has one; none has two while another has none
  p.clusters = (int)std::min<int64_t>(sms / q.ctas, (int64_t)d->n_replicas * q.m_tiles * p.n_units);
  const int lists = list_bytes(q.held);
  p.stages = std::min(kMaxStages, (kMaxSmem - kFixedSmem - lists) / kStageBytes);
  const int smem = kFixedSmem + lists + p.stages * kStageBytes;
  const auto kernel = q.ctas == 1 ? pick_kernel<1>(q.held) : pick_kernel<2>(q.held);
  e = launch(kernel, dim3((unsigned)(p.clusters * q.ctas)), kScoreThreads, smem, q.ctas, st, p);
  if (e == cudaSuccess) {
    const int64_t rows = d->n_replicas * d->n_tokens;
    const int warps = rows <= kFewRowsToJoin ? 32 : rows < kManyRows ? 8 : 1;
    const auto of = [&](auto few, auto some, auto many) { return join(warps == 32 ? few : warps == 8 ? some : many, warps); };
    if (q.held == kKeep)
      e = q.ctas == 1 ? of(join_scores_kernel<1, 32, true>, join_scores_kernel<1, 8, true>, join_scores_kernel<1, 1, true>)
                      : of(join_scores_kernel<2, 32, true>, join_scores_kernel<2, 8, true>, join_scores_kernel<2, 1, true>);
    else
      e = q.ctas == 1 ? of(join_scores_kernel<1, 32>, join_scores_kernel<1, 8>, join_scores_kernel<1, 1>)
                      : of(join_scores_kernel<2, 32>, join_scores_kernel<2, 8>, join_scores_kernel<2, 1>);
  }
  return e == cudaSuccess ? HDET_OK : fail_cuda(who, e);
}

}  // namespace
}  // namespace hdet

using namespace hdet;

extern "C" HDET_API int hdet_token_scores_workspace(const hdet_token_scores_args* d, int64_t* bytes) {
  const char* who = "hdet_token_scores_workspace";
  if (!bytes) return fail(HDET_ERR_INVALID_ARG, who, "bytes is NULL");
  *bytes = 0;
  if (const int rc = check_token_scores(who, d, false)) return rc;
  *bytes = workspace_of(d);
  return HDET_OK;
}

extern "C" HDET_API int hdet_token_scores(const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return token_scores("hdet_token_scores", d, workspace, workspace_bytes, stream, false);
}

extern "C" HDET_API int hdet_selftest_token_scores_wait(const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return token_scores("hdet_selftest_token_scores_wait", d, workspace, workspace_bytes, stream, true);
}
