// Embedding lookup with scaling, and its gradient by sorted tokens (contract: include/hdet.h).
//
//   lookup    rows[r,t,:] = scale * table[r, tok[r,t], :]
//   gradient  table[r,v,:] (+)= scale * sum over t with tok[r,t] = v of rows[r,t,:]
//
// Both are bound by HBM.  The gradient is a sum over tokens that share a row.  Atomics would add them in an order
// that changes from run to run, so the tokens are sorted first (stable: equal tokens stay in the order of t) and every
// row is summed in that order in fp32 by one owner, then rounded once.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "hdet_internal.h"
#include "hdet_launch.cuh"
#include "../../include/hdet.h"

namespace {

using hdet::launch;
using hdet::let_next_start;
using hdet::wait_for_previous;

constexpr int kChunk = 1024;        // tokens sorted by one block
constexpr int kMergeRuns = 8;       // sorted runs merged per level
constexpr int kEntries = 32;        // sorted entries per warp in the gradient kernel, one per lane
constexpr int kFewEntries = 8;      // ... when there are too few to keep the machine busy: one batch of loads each

__host__ __device__ constexpr int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Token t of replica r as a row index; anything outside 0 .. vocab-1 becomes vocab, "no row".
__device__ __forceinline__ int row_of(const void* tokens, bool wide, int64_t at, int vocab) {
  if (wide) {
    const long long v = static_cast<const long long*>(tokens)[at];
    return v >= 0 && v < vocab ? (int)v : vocab;
  }
  const int v = static_cast<const int*>(tokens)[at];
  return v >= 0 && v < vocab ? v : vocab;
}

// VEC consecutive elements of type T, moved in accesses of at most 16 bytes; VEC * sizeof(T) bytes aligned (16 at most).
template <typename T, int VEC>
struct Pack {
  static constexpr int kBytes = VEC * (int)sizeof(T);
  static constexpr int kAlign = kBytes < 16 ? kBytes : 16;
  struct alignas(kAlign) Raw { T v[VEC]; };
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return raw.v[i]; else return __bfloat162float(raw.v[i]);
  }
  __device__ __forceinline__ void set(int i, float x) {
    if constexpr (sizeof(T) == 4) raw.v[i] = x; else raw.v[i] = __float2bfloat16_rn(x);
  }
};

struct EmbedParams {
  const void* tokens;
  void* rows;
  void* table;
  int64_t token_stride, rows_stride, rows_row, table_stride, table_row;
  int64_t n_tokens, width;
  int vocab, n_replicas;
  bool wide;
  float scale;
};

// ------------------------------------------------------------------------------------------------ lookup
// A block covers blockDim.y rows times kRowsPerThread, and blockDim.x vectors of each; every thread reads its
// kRowsPerThread token ids, then has that many independent row loads in flight.
constexpr int kRowsPerThread = 4;

template <typename TableT, typename RowT, int VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const EmbedParams p) {
  let_next_start();
  wait_for_previous();
  const int64_t base = (int64_t)blockIdx.x * (blockDim.y * kRowsPerThread) + threadIdx.y;
  const int r = blockIdx.y;
  const TableT* table = static_cast<const TableT*>(p.table) + r * p.table_stride;
  RowT* rows = static_cast<RowT*>(p.rows) + r * p.rows_stride;
  int id[kRowsPerThread];
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int64_t t = base + (int64_t)k * blockDim.y;
    id[k] = t < p.n_tokens ? row_of(p.tokens, p.wide, r * p.token_stride + t, p.vocab) : -1;
  }
  for (int64_t c = (int64_t)threadIdx.x * VEC; c < p.width; c += (int64_t)blockDim.x * VEC) {
    Pack<TableT, VEC> x[kRowsPerThread];
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k)
      if (id[k] >= 0 && id[k] < p.vocab) x[k].load(table + id[k] * p.table_row + c);
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
      if (id[k] < 0) continue;
      const bool some = id[k] < p.vocab;
      Pack<RowT, VEC> y;
#pragma unroll
      for (int i = 0; i < VEC; ++i) y.set(i, some ? x[k].get(i) * p.scale : 0.0f);
      y.store(rows + (base + (int64_t)k * blockDim.y) * p.rows_row + c);
    }
  }
}

// ------------------------------------------------------------------------------------------------ sorting
// Entries of run[0 .. n) that come before `key`: those < key, or <= key.
__device__ __forceinline__ int64_t count_before(const int* __restrict__ run, int64_t n, int key, bool or_equal) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    const int o = run[mid];
    if (o < key || (or_equal && o == key)) lo = mid + 1; else hi = mid;
  }
  return lo;
}

// Sorts 1024 tokens a block, one a thread: 32 in a warp by comparing each with all, then runs of 32, 64, .. 512 are merged in
// pairs, where an entry's place is its place in its own run plus the entries of the other run that come before it (a binary
// search in shared memory).  Equal tokens keep their order: of the run before, those that are equal count too.
// Comparing all 1024 with one another instead took 13.3 us for 8 x 8192 tokens, this takes 6.1 us.
__global__ void __launch_bounds__(kChunk) sort_chunks_kernel(const EmbedParams p, int* __restrict__ key_out, int* __restrict__ pos_out) {
  __shared__ int s_key[2][kChunk], s_from[2][kChunk];
  let_next_start();
  wait_for_previous();
  const int r = blockIdx.y, i = threadIdx.x, lane = i & 31;
  const int64_t c0 = (int64_t)blockIdx.x * kChunk;
  // entries behind the end compare as larger than every row and than "no row"
  int key = c0 + i < p.n_tokens ? row_of(p.tokens, p.wide, r * p.token_stride + c0 + i, p.vocab) : 0x7fffffff;
  int from = i, place = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const int o = __shfl_sync(0xffffffffu, key, j);
    place += o < key || (o == key && j < lane);
  }
  place += i - lane;
  int now = 0;
  s_key[0][place] = key;
  s_from[0][place] = from;
  __syncthreads();
#pragma unroll
  for (int run = 32; run < kChunk; run *= 2) {
    key = s_key[now][i];
    from = s_from[now][i];
    const bool second = i & run;
    const int* other = s_key[now] + ((i & ~(run - 1)) ^ run);
    int before = 0;                                // entries of the other run that come before this one
#pragma unroll
    for (int step = run; step > 0; step /= 2) {
      if (before + step > run) continue;
      const int o = other[before + step - 1];
      if (o < key || (o == key && second)) before += step;
    }
    place = (i & ~(2 * run - 1)) + (i & (run - 1)) + before;
    now ^= 1;
    s_key[now][place] = key;
    s_from[now][place] = from;
    __syncthreads();
  }
  if (c0 + i < p.n_tokens) {
    key_out[r * p.n_tokens + c0 + i] = s_key[now][i];
    pos_out[r * p.n_tokens + c0 + i] = (int)c0 + s_from[now][i];
  }
}

// Merges groups of kMergeRuns sorted runs of `run` (a power of two) entries: an entry's place in its group is its place in
// its own run plus, for every other run, the entries there that come before it.  The searches in the other runs go step by
// step together, so that their loads are under way at once.
__global__ void __launch_bounds__(256) merge_runs_kernel(int64_t n, int64_t run, const int* __restrict__ key_in,
                                                         const int* __restrict__ pos_in, int* __restrict__ key_out,
                                                         int* __restrict__ pos_out) {
  let_next_start();
  wait_for_previous();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int64_t base = (int64_t)blockIdx.y * n;
  const int* keys = key_in + base;
  const int key = keys[i], pos = pos_in[base + i];
  const int64_t own = i / run, first = own / kMergeRuns * kMergeRuns;
  int before[kMergeRuns];                          // entries of each run found to come before this one
#pragma unroll
  for (int q = 0; q < kMergeRuns; ++q) before[q] = 0;
  for (int64_t step = run; step > 0; step >>= 1) {
    int o[kMergeRuns];                             // the last of each run's next `step` entries
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q) {
      const int64_t at = (first + q) * run + before[q] + step - 1;
      o[q] = before[q] + step <= run && at < n && first + q != own ? keys[at] : 0x7fffffff;
    }
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q)
      if (o[q] < key || (o[q] == key && first + q < own)) before[q] += (int)step;
  }
  int64_t at = first * run + (i - own * run);
#pragma unroll
  for (int q = 0; q < kMergeRuns; ++q) at += before[q];
  key_out[base + at] = key;
  pos_out[base + at] = pos;
}

// ------------------------------------------------------------------------------------------------ gradient
struct GradParams {
  EmbedParams e;
  const int* keys;       // [replicas or 1][n_tokens], sorted; vocab = no row
  const int* pos;        // the token behind each key
  int64_t sorted_stride; // n_tokens, or 0 when all replicas share one batch of tokens
  float* partial;        // [replicas][blocks][2][width]
  int64_t n_blocks;      // entry blocks per replica
  int64_t n_col;         // column chunks of 32 * VEC
  int64_t grad_units;    // n_blocks * n_col
  int64_t zero_units;    // 32-row groups of the table to look at for rows without a token (0 when accumulating)
  unsigned grad_ctas, zero_ctas;
  int entries;           // sorted entries per block: kEntries or kFewEntries
  bool accumulate;
};

template <typename TableT, int VEC>
__device__ __forceinline__ void write_row(const GradParams& p, int r, int key, int64_t c, const float (&acc)[VEC]) {
  TableT* to = static_cast<TableT*>(p.e.table) + r * p.e.table_stride + key * p.e.table_row + c;
  Pack<TableT, VEC> y;
  if (p.accumulate) {
    y.load(to);
#pragma unroll
    for (int i = 0; i < VEC; ++i) y.set(i, fmaf(acc[i], p.e.scale, y.get(i)));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) y.set(i, acc[i] * p.e.scale);
  }
  y.store(to);
}

// One warp: an entry block of `entries` consecutive sorted entries (one per lane) and 32 * VEC columns.  A run of equal keys
// that lies inside the block is finished here; the piece of a run that came from the block before goes to partial slot 0, the piece
// of a run that starts here and goes on into the next block to slot 1, and join_kernel adds those in order.
// Other warps write zeros to the table rows that have no token.  The two kinds of blocks alternate in the grid, in proportion,
// so that the sums' loads hide behind the zeros' stores (8 x 8192 tokens, width 2048: 1.5 % less than the zeros behind the sums).
//
// With ADD, the table's rows that a batch of entries will finish are loaded along with the entries' own: loaded one by one at
// the end of each run they took 141 us for that batch, with this it is 122 us.
template <typename RowT, typename TableT, int VEC, bool ADD>
__global__ void __launch_bounds__(256) grad_kernel(const GradParams p) {
  // The next kernel is not let in early here: with that, 16 x 1024 tokens of width 768 took 249 us instead of 215 (why is not known; the
  // next kernel starts when every block of this one has started or ended).
  wait_for_previous();
  const int r = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t n = p.e.n_tokens;
  const int* keys = p.keys + r * p.sorted_stride;
  // of the first b blocks, b * grad_ctas / all (rounded down) are for sums
  const uint64_t all = (uint64_t)p.grad_ctas + p.zero_ctas;
  const uint64_t sums_before = (uint64_t)blockIdx.x * p.grad_ctas / all;
  const bool sums = (uint64_t)(blockIdx.x + 1) * p.grad_ctas / all > sums_before;
  const int64_t unit = (int64_t)(sums ? sums_before : blockIdx.x - sums_before) * 8 + (threadIdx.x >> 5);
  if (!sums) {
    const int64_t row0 = unit * 32;
    if (unit >= p.zero_units) return;
    bool empty = false;
    if (row0 + lane < p.e.vocab) {
      const int64_t at = count_before(keys, n, (int)(row0 + lane), false);
      empty = at >= n || keys[at] != row0 + lane;
    }
    unsigned todo = __ballot_sync(0xffffffffu, empty);
    // at most 16 bytes a thread, so that every store of the warp is whole lines (fp32 table of 14 x 33848 x 512, all zeros but
    // for a few rows: 161 us; in two stores of 16 bytes a thread 32 apart 197)
    constexpr int kWide = VEC * (int)sizeof(TableT) > 16 ? 16 / (int)sizeof(TableT) : VEC;
    Pack<TableT, kWide> zero;
#pragma unroll
    for (int i = 0; i < kWide; ++i) zero.set(i, 0.0f);
    TableT* table = static_cast<TableT*>(p.e.table) + r * p.e.table_stride;
    for (; todo; todo &= todo - 1) {
      TableT* row = table + (row0 + __ffs(todo) - 1) * p.e.table_row;
      for (int64_t c = (int64_t)lane * kWide; c < p.e.width; c += 32 * kWide) zero.store(row + c);
    }
    return;
  }
  if (unit >= p.grad_units) return;
  const int64_t block = unit / p.n_col;
  const int64_t c = (unit % p.n_col) * (32 * VEC) + (int64_t)lane * VEC;
  const bool on = c < p.e.width;
  const int64_t i0 = block * p.entries;
  const int* pos = p.pos + r * p.sorted_stride;
  const bool mine = lane < p.entries && i0 + lane < n;
  const int my_key = mine ? keys[i0 + lane] : p.e.vocab;
  const int my_pos = mine ? pos[i0 + lane] : 0;
  const int before = i0 > 0 ? keys[i0 - 1] : -1;
  const int after = i0 + p.entries < n ? keys[i0 + p.entries] : p.e.vocab;
  const int count = __popc(__ballot_sync(0xffffffffu, my_key < p.e.vocab));   // sorted: the entries with a row come first
  const RowT* rows = static_cast<const RowT*>(p.e.rows) + r * p.e.rows_stride;
  float* partial = p.partial + ((int64_t)r * p.n_blocks + block) * 2 * p.e.width;
  float acc[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
  bool from_before = false;
  constexpr int kAhead = ADD ? 4 : 8;
  TableT* table = static_cast<TableT*>(p.e.table) + r * p.e.table_stride;
  for (int e0 = 0; e0 < count; e0 += kAhead) {
    Pack<RowT, VEC> x[kAhead];
    Pack<TableT, VEC> old[ADD ? kAhead : 1];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int ps = __shfl_sync(0xffffffffu, my_pos, (e0 + k) & 31);
      if (e0 + k < count && on) x[k].load(rows + ps * p.e.rows_row + c);
      if constexpr (ADD) {
        const int key = __shfl_sync(0xffffffffu, my_key, (e0 + k) & 31), next = __shfl_sync(0xffffffffu, my_key, (e0 + k + 1) & 31);
        if (e0 + k < count && on && (next != key || e0 + k + 1 == p.entries)) old[k].load(table + key * p.e.table_row + c);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = e0 + k;
      if (e >= count) break;
      const int key = __shfl_sync(0xffffffffu, my_key, e);
      const int next_lane = __shfl_sync(0xffffffffu, my_key, (e + 1) & 31);
      const int next = e + 1 < p.entries ? next_lane : after;
      if (e == 0) from_before = key == before;
      if (on) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += x[k].get(i);
      }
      if (next == key && e + 1 < p.entries) continue;
      // the run's piece in this block ends here
      const bool goes_on = e + 1 == p.entries && next == key;
      if (on) {
        if (from_before || goes_on) {
          float* to = partial + (from_before ? 0 : p.e.width) + c;
#pragma unroll
          for (int i = 0; i < VEC; ++i) to[i] = acc[i];
        } else {
          Pack<TableT, VEC> y;
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            if constexpr (ADD) y.set(i, fmaf(acc[i], p.e.scale, old[k].get(i)));
            else y.set(i, acc[i] * p.e.scale);
          }
          y.store(table + key * p.e.table_row + c);
        }
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
      from_before = false;
    }
  }
}

// The runs that start in an entry block and go on behind it: their pieces are added in order.  A block of threads looks at 32
// entry blocks and one column chunk; every run found is one warp's, and a run of more than kLongRun pieces is shared by all
// eight, which take consecutive stretches whose sums are added in order, so no result depends on timing.
constexpr int kLongRun = 64, kJoinBlocks = 32;

template <int VEC>
__device__ __forceinline__ void add_pieces(const float* first, int64_t width, int64_t from, int64_t to, float (&acc)[VEC]) {
  // piece 0 is slot 1 of the run's first block, piece j > 0 slot 0 of the j-th behind it
#pragma unroll 8
  for (int64_t j = from; j < to; ++j) {
    const float* x = first + (j == 0 ? width : j * 2 * width);
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] += x[i];
  }
}

template <typename TableT, int VEC>
__global__ void __launch_bounds__(256) join_kernel(const GradParams p) {
  __shared__ float s_sum[8][32 * VEC];
  let_next_start();
  wait_for_previous();
  const int r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t block0 = (int64_t)(blockIdx.x / p.n_col) * kJoinBlocks;
  const int64_t c = (blockIdx.x % p.n_col) * (32 * VEC) + (int64_t)lane * VEC;
  const bool on = c < p.e.width;
  const int64_t n = p.e.n_tokens;
  const int* keys = p.keys + r * p.sorted_stride;
  // lane l of every warp: does a run start in entry block block0 + l and go on behind it
  const int64_t i0 = (block0 + lane) * p.entries, next = i0 + p.entries;
  int key = p.e.vocab, head = p.e.vocab, after = -1;   // the block's last and first key, the next block's first
  bool runs = false;
  if (i0 < n) {
    head = keys[i0];
    if (next < n) {
      key = keys[next - 1];
      after = keys[next];
      runs = key < p.e.vocab && after == key && !(i0 > 0 && head == key && keys[i0 - 1] == key);
    }
  }
  // Of how many pieces: the blocks here whose first key is the run's.  Only one run can go on behind these 32 blocks: its end
  // is searched for.
  const int beyond = __shfl_sync(0xffffffffu, after, 31);
  const unsigned all = __ballot_sync(0xffffffffu, runs);
  int64_t pieces = 0;
  for (unsigned todo = all; todo; todo &= todo - 1) {
    const int l = __ffs(todo) - 1, row = __shfl_sync(0xffffffffu, key, l);
    const unsigned on_from = __ballot_sync(0xffffffffu, head == row && lane > l);
    if (lane == l) pieces = 1 + __popc(on_from);
  }
  if (__any_sync(0xffffffffu, runs && key == beyond)) {   // 32 blocks at a time, then by halves
    int64_t more = 0;
    bool whole = true;
    for (int step = 0; step < 4 && whole; ++step) {
      const int64_t at = (block0 + 32 * (step + 1) + lane) * p.entries;
      const unsigned same = __ballot_sync(0xffffffffu, at < n && keys[at] == beyond);
      more += __popc(same);
      whole = same == 0xffffffffu;
    }
    if (whole) {
      const int64_t at = (block0 + 32 * 5) * p.entries;
      more += at < n ? div_up(count_before(keys + at, n - at, beyond, true), p.entries) : 0;
    }
    if (runs && key == beyond) pieces += more;
  }
  const unsigned shared_runs = __ballot_sync(0xffffffffu, pieces > kLongRun);
  float acc[VEC];
  int turn = 0;
  for (unsigned todo = all & ~shared_runs; todo; todo &= todo - 1, ++turn) {
    if (turn % 8 != warp) continue;
    const int l = __ffs(todo) - 1;
    const int64_t count = __shfl_sync(0xffffffffu, pieces, l);
    const int row = __shfl_sync(0xffffffffu, key, l);
    if (!on) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    add_pieces<VEC>(p.partial + ((int64_t)r * p.n_blocks + block0 + l) * 2 * p.e.width + c, p.e.width, 0, count, acc);
    write_row<TableT, VEC>(p, r, row, c, acc);
  }
  for (unsigned todo = shared_runs; todo; todo &= todo - 1) {
    const int l = __ffs(todo) - 1;
    const int64_t count = __shfl_sync(0xffffffffu, pieces, l), each = div_up(count, 8);
    const int row = __shfl_sync(0xffffffffu, key, l);
    const int64_t from = warp * each, to = from + each < count ? from + each : count;
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.0f;
    if (on) add_pieces<VEC>(p.partial + ((int64_t)r * p.n_blocks + block0 + l) * 2 * p.e.width + c, p.e.width, from, to, acc);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s_sum[warp][i * 32 + lane] = acc[i];
    __syncthreads();
    if (warp == 0 && on) {
      for (int w = 1; w < 8; ++w)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += s_sum[w][i * 32 + lane];
      write_row<TableT, VEC>(p, r, row, c, acc);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ host side
int fail(int code, const char* who, const char* what) {
  char msg[240];
  snprintf(msg, sizeof msg, "%s: %s", who, what);
  hdet::set_handleless_error(msg);
  return code;
}

int elem_size(int dtype) { return dtype == HDET_DTYPE_BF16 ? 2 : 4; }

// Checks shared by the three entry points.
int check(const char* who, const hdet_embedding* d) {
  if (!d) return fail(HDET_ERR_INVALID_ARG, who, "the descriptor is NULL");
  if (d->n_replicas < 1 || d->n_replicas > HDET_MAX_REPLICAS)
    return fail(HDET_ERR_INVALID_ARG, who, "n_replicas must be in 1..32");
  if (d->n_tokens < 0 || d->n_tokens > HDET_MAX_TOKENS || d->vocab < 1 || d->vocab > HDET_MAX_VOCAB || d->width < 1 ||
      d->width > HDET_MAX_WIDTH)
    return fail(HDET_ERR_INVALID_ARG, who, "n_tokens, vocab or width out of range");
  if (d->token_dtype != HDET_DTYPE_I32 && d->token_dtype != HDET_DTYPE_I64)
    return fail(HDET_ERR_INVALID_ARG, who, "token_dtype must be HDET_DTYPE_I32 or HDET_DTYPE_I64");
  if ((d->table_dtype != HDET_DTYPE_F32 && d->table_dtype != HDET_DTYPE_BF16) ||
      (d->rows_dtype != HDET_DTYPE_F32 && d->rows_dtype != HDET_DTYPE_BF16))
    return fail(HDET_ERR_INVALID_ARG, who, "table_dtype and rows_dtype must be HDET_DTYPE_F32 or HDET_DTYPE_BF16");
  if (d->device < 0) return fail(HDET_ERR_INVALID_ARG, who, "device must be >= 0");
  if (!std::isfinite((float)d->scale)) return fail(HDET_ERR_INVALID_ARG, who, "scale must be finite in fp32");
  if (d->table_row < d->width || d->rows_row < d->width)
    return fail(HDET_ERR_INVALID_ARG, who, "a row stride is smaller than width");
  if (std::max(d->table_row, d->rows_row) > HDET_MAX_ROW_STRIDE)
    return fail(HDET_ERR_INVALID_ARG, who, "a row stride is out of range");
  if (d->n_replicas > 1 && std::max({d->table_stride, d->rows_stride, d->token_stride}) > HDET_MAX_REPLICA_STRIDE)
    return fail(HDET_ERR_INVALID_ARG, who, "a replica stride is out of range");
  return HDET_OK;
}

// Checks of the pointers, and of strides that the call will write through.
int check_pointers(const char* who, const hdet_embedding* d, bool writes_table) {
  if (!d->table || (d->n_tokens > 0 && (!d->tokens || !d->rows)))
    return fail(HDET_ERR_INVALID_ARG, who, "a pointer is NULL");
  const int64_t table_len = (d->vocab - 1) * d->table_row + d->width;
  const int64_t rows_len = d->n_tokens > 0 ? (d->n_tokens - 1) * d->rows_row + d->width : 0;
  if (d->n_replicas > 1) {
    if (d->table_stride < 0 || d->rows_stride < 0 || d->token_stride < 0)
      return fail(HDET_ERR_INVALID_ARG, who, "negative stride");
    if (d->table_stride < table_len && (writes_table || d->table_stride != 0))
      return fail(HDET_ERR_INVALID_ARG, who, "table_stride is smaller than one table");
    if (d->rows_stride < rows_len && (!writes_table || d->rows_stride != 0))
      return fail(HDET_ERR_INVALID_ARG, who, "rows_stride is smaller than one replica's rows");
    if (d->token_stride < d->n_tokens && d->token_stride != 0)
      return fail(HDET_ERR_INVALID_ARG, who, "token_stride is smaller than n_tokens");
  }
  const uintptr_t a = reinterpret_cast<uintptr_t>(d->tokens) % (d->token_dtype == HDET_DTYPE_I64 ? 8 : 4);
  const uintptr_t b = reinterpret_cast<uintptr_t>(d->table) % elem_size(d->table_dtype);
  const uintptr_t c = reinterpret_cast<uintptr_t>(d->rows) % elem_size(d->rows_dtype);
  if (a || b || c) return fail(HDET_ERR_ALIGN, who, "a pointer is not aligned to its element type");
  return HDET_OK;
}

EmbedParams params_of(const hdet_embedding* d) {
  EmbedParams p{};
  p.tokens = d->tokens; p.rows = d->rows; p.table = d->table;
  const bool many = d->n_replicas > 1;
  p.token_stride = many ? d->token_stride : 0;
  p.rows_stride = many ? d->rows_stride : 0;
  p.table_stride = many ? d->table_stride : 0;
  p.rows_row = d->rows_row; p.table_row = d->table_row;
  p.n_tokens = d->n_tokens; p.width = d->width; p.vocab = (int)d->vocab; p.n_replicas = d->n_replicas;
  p.wide = d->token_dtype == HDET_DTYPE_I64;
  p.scale = (float)d->scale;
  return p;
}

// Elements per access: the largest of 8, 4, 2, 1 that divides the width and every stride and keeps each access inside
// one aligned 16-byte unit (or whole units) on both sides.
int vector_of(const hdet_embedding* d) {
  const bool many = d->n_replicas > 1;
  for (int v = 8; v > 1; v /= 2) {
    if (d->width % v || d->rows_row % v || d->table_row % v) continue;
    if (many && (d->rows_stride % v || d->table_stride % v)) continue;
    const int rb = v * elem_size(d->rows_dtype), tb = v * elem_size(d->table_dtype);
    if (reinterpret_cast<uintptr_t>(d->rows) % (rb < 16 ? rb : 16)) continue;
    if (reinterpret_cast<uintptr_t>(d->table) % (tb < 16 ? tb : 16)) continue;
    return v;
  }
  return 1;
}

// Sets the descriptor's device for the scope of one call and restores the caller's.
struct DeviceScope {
  int prev = -1;
  bool switched = false;
  cudaError_t err = cudaSuccess;
  explicit DeviceScope(int dev) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != dev) {
      err = cudaSetDevice(dev);
      switched = err == cudaSuccess;
    }
  }
  ~DeviceScope() { if (switched) cudaSetDevice(prev); }
};

// The call's own error, which does not stay behind for whoever asks the runtime for its last one next.
int fail_cuda(const char* who, cudaError_t e) {
  cudaGetLastError();
  return fail(HDET_ERR_CUDA, who, cudaGetErrorString(e));
}

template <typename TableT, typename RowT, int VEC>
cudaError_t launch_lookup(const EmbedParams& p, cudaStream_t st) {
  int x = 1;
  while (x < 256 && (int64_t)x * VEC < p.width) x *= 2;
  const dim3 block(x, 256 / x);
  const dim3 grid((unsigned)div_up(p.n_tokens, (int64_t)block.y * kRowsPerThread), p.n_replicas);
  return launch(lookup_kernel<TableT, RowT, VEC>, grid, block, 0, 1, st, p);
}

template <typename RowT, typename TableT, int VEC>
cudaError_t launch_grad(GradParams p, cudaStream_t st) {
  p.n_blocks = div_up(p.e.n_tokens, p.entries);
  p.n_col = div_up(p.e.width, 32 * VEC);
  p.grad_units = p.n_blocks * p.n_col;
  p.zero_units = p.accumulate ? 0 : div_up(p.e.vocab, 32);
  p.grad_ctas = (unsigned)div_up(p.grad_units, 8);
  p.zero_ctas = (unsigned)div_up(p.zero_units, 8);
  cudaError_t e = cudaSuccess;
  if (p.grad_ctas + p.zero_ctas > 0)
    e = launch(p.accumulate ? grad_kernel<RowT, TableT, VEC, true> : grad_kernel<RowT, TableT, VEC, false>,
               dim3(p.grad_ctas + p.zero_ctas, p.e.n_replicas), 256, 0, 1, st, p);
  if (e == cudaSuccess && p.n_blocks > 1)
    e = launch(join_kernel<TableT, VEC>, dim3((unsigned)(div_up(p.n_blocks, kJoinBlocks) * p.n_col), p.e.n_replicas), 256, 0, 1, st, p);
  return e;
}

// Calls f.template operator()<A, B, VEC>() for the element types and the vector width.
template <typename A, typename B, typename F>
void with_vector(int vec, F&& f) {
  if (vec == 8) f.template operator()<A, B, 8>();
  else if (vec == 4) f.template operator()<A, B, 4>();
  else if (vec == 2) f.template operator()<A, B, 2>();
  else f.template operator()<A, B, 1>();
}

template <typename F>
void with_types(int a, int b, int vec, F&& f) {
  if (a == HDET_DTYPE_F32 && b == HDET_DTYPE_F32) with_vector<float, float>(vec, f);
  else if (a == HDET_DTYPE_F32) with_vector<float, __nv_bfloat16>(vec, f);
  else if (b == HDET_DTYPE_F32) with_vector<__nv_bfloat16, float>(vec, f);
  else with_vector<__nv_bfloat16, __nv_bfloat16>(vec, f);
}

struct LookupLauncher {
  const EmbedParams& p;
  cudaStream_t st;
  cudaError_t err = cudaSuccess;
  template <typename TableT, typename RowT, int VEC> void operator()() { err = launch_lookup<TableT, RowT, VEC>(p, st); }
};

struct GradLauncher {
  const GradParams& p;
  cudaStream_t st;
  cudaError_t err = cudaSuccess;
  template <typename RowT, typename TableT, int VEC> void operator()() { err = launch_grad<RowT, TableT, VEC>(p, st); }
};

// Workspace of the gradient: two copies of the sorted keys and positions, then the partial sums.
struct GradLayout {
  int64_t list_bytes;     // one array of one entry per sorted token
  int64_t partial_off, total;
  int sorted_replicas, entries;
};

// Up to how many tokens the gradient kernel has fewer than 4 x 148 warps with long entry blocks.
int64_t few_tokens(const hdet_embedding* d) { return (4 * 148 - 1) / (div_up(d->width, 256) * d->n_replicas) * kEntries; }

GradLayout layout_of(const hdet_embedding* d, int64_t n_tokens) {
  GradLayout l{};
  const auto up = [](int64_t x) { return div_up(x, 256) * 256; };
  l.sorted_replicas = d->n_replicas > 1 && d->token_stride != 0 ? d->n_replicas : 1;
  // Fewer than four warps a SM in the gradient kernel: shorter entry blocks make more of them (96 tokens of
  // width 72: 6.8 us instead of 8.6).
  l.entries = n_tokens <= few_tokens(d) ? kFewEntries : kEntries;
  l.list_bytes = up(4 * n_tokens * l.sorted_replicas);
  l.partial_off = 4 * l.list_bytes;
  l.total = l.partial_off + up(4 * 2 * d->width * div_up(n_tokens, l.entries) * d->n_replicas);
  if (l.total < 256) l.total = 256;
  return l;
}

// The most that a call with up to n_tokens tokens needs: the last batch with short entry blocks has more partial sums than the first with
// long ones.
int64_t workspace_of(const hdet_embedding* d) {
  return std::max(layout_of(d, d->n_tokens).total, layout_of(d, std::min(d->n_tokens, few_tokens(d))).total);
}

}  // namespace

extern "C" HDET_API int hdet_embed(const hdet_embedding* d, void* stream) {
  hdet::TraceRange trace("hdet_embed");
  if (const int rc = check("hdet_embed", d)) return rc;
  if (const int rc = check_pointers("hdet_embed", d, false)) return rc;
  if (d->n_tokens == 0) return HDET_OK;
  DeviceScope scope(d->device);
  if (scope.err != cudaSuccess) return fail_cuda("hdet_embed", scope.err);
  const EmbedParams p = params_of(d);
  LookupLauncher launcher{p, static_cast<cudaStream_t>(stream)};
  with_types(d->table_dtype, d->rows_dtype, vector_of(d), launcher);
  return launcher.err == cudaSuccess ? HDET_OK : fail_cuda("hdet_embed", launcher.err);
}

extern "C" HDET_API int hdet_embed_grad_workspace(const hdet_embedding* d, int64_t* bytes) {
  if (!bytes) return fail(HDET_ERR_INVALID_ARG, "hdet_embed_grad_workspace", "bytes is NULL");
  *bytes = 0;
  if (const int rc = check("hdet_embed_grad_workspace", d)) return rc;
  *bytes = workspace_of(d);
  return HDET_OK;
}

extern "C" HDET_API int hdet_embed_grad(const hdet_embedding* d, int32_t accumulate, void* workspace,
                                        int64_t workspace_bytes, void* stream) {
  hdet::TraceRange trace("hdet_embed_grad");
  if (const int rc = check("hdet_embed_grad", d)) return rc;
  if (const int rc = check_pointers("hdet_embed_grad", d, true)) return rc;
  const GradLayout l = layout_of(d, d->n_tokens);
  if (!workspace || workspace_bytes < l.total)
    return fail(HDET_ERR_INVALID_ARG, "hdet_embed_grad", "the workspace is NULL or smaller than hdet_embed_grad_workspace says");
  if (reinterpret_cast<uintptr_t>(workspace) % 256)
    return fail(HDET_ERR_ALIGN, "hdet_embed_grad", "the workspace is not 256-byte aligned");
  DeviceScope scope(d->device);
  if (scope.err != cudaSuccess) return fail_cuda("hdet_embed_grad", scope.err);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  int *key[2], *pos[2];
  for (int k = 0; k < 2; ++k) {
    key[k] = reinterpret_cast<int*>(ws + k * l.list_bytes);
    pos[k] = reinterpret_cast<int*>(ws + (2 + k) * l.list_bytes);
  }
  const EmbedParams e = params_of(d);
  int now = 0;
  if (d->n_tokens > 0) {
    cudaError_t err = launch(sort_chunks_kernel, dim3((unsigned)div_up(d->n_tokens, kChunk), l.sorted_replicas), kChunk, 0, 1, st, e,
                             key[0], pos[0]);
    for (int64_t run = kChunk; run < d->n_tokens && err == cudaSuccess; run *= kMergeRuns, now ^= 1)
      err = launch(merge_runs_kernel, dim3((unsigned)div_up(d->n_tokens, 256), l.sorted_replicas), 256, 0, 1, st, d->n_tokens, run,
                   key[now], pos[now], key[now ^ 1], pos[now ^ 1]);
    if (err != cudaSuccess) return fail_cuda("hdet_embed_grad", err);
  }
  GradParams p{};
  p.e = e;
  p.keys = key[now];
  p.pos = pos[now];
  p.sorted_stride = l.sorted_replicas > 1 ? d->n_tokens : 0;
  p.partial = reinterpret_cast<float*>(ws + l.partial_off);
  p.accumulate = accumulate != 0;
  p.entries = l.entries;
  GradLauncher launcher{p, st};
  with_types(d->rows_dtype, d->table_dtype, vector_of(d), launcher);
  return launcher.err == cudaSuccess ? HDET_OK : fail_cuda("hdet_embed_grad", launcher.err);
}
