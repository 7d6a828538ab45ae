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
//   scores   a CTA (or pair) takes 128 (256) tokens and a run of the vocabulary's tiles, one after the other: a reader keeps its row's
//            state and its list of the best classes over the whole run
//   join     a block a row: the runs' states and lists become the row's; the best are summed again in fp64 and ordered
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
constexpr int kGroup = 16;                 // columns that are looked through at a time for a list
constexpr int kMaxSmem = 227 * 1024;
constexpr long long kSelftestLimitCycles = 4000000ll;   // 2 ms
constexpr int kChunk = 16;                 // steps of 64 that the tensor cores sum before fp32 registers take over, as in the loss

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

// A row's state over some of its classes.
struct State {
  float top, others, weighted, ties;       // M, delta, U, n
  __device__ __forceinline__ void clear() { top = -INFINITY; others = weighted = ties = 0.0f; }
  // Moves the reference up to `to` > top: those that had the maximum are others now.
  __device__ __forceinline__ void raise(float to) {
    const float d = top - to, f = exp_from(top, to), all = ties + others;
    if (all != 0.0f) {                     // (not for the first value, where top is -inf)
      weighted = f * fmaf(all, d, weighted);
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
  __device__ __forceinline__ void add_logit(float z) {
    if (z > top) raise(z);
    if (z == top) {
      ties += z > -INFINITY;
    } else {
      const float d = z - top, e = exp_from(z, top);
      others += e;
      weighted = fmaf(e, fmaxf(d, -1e4f), weighted);       // a logit of -inf adds 0, not NaN; one that is NaN makes others NaN
    }
  }
  __device__ __forceinline__ void add_lane(int o) {
    State s;
    s.top = __shfl_xor_sync(0xffffffffu, top, o);
    s.others = __shfl_xor_sync(0xffffffffu, others, o);
    s.weighted = __shfl_xor_sync(0xffffffffu, weighted, o);
    s.ties = __shfl_xor_sync(0xffffffffu, ties, o);
    add(s);
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
  Key* lists;               // scores: [job][half][entry][row of the tile]; few: [replica][token][part][entry]
  Key* best;                // a list's first, laid out as part
  int n_parts;              // few: blocks a replica
  int n_tiles;              // of the vocabulary
  int list;                 // entries of a list, 0: none
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

// How many runs the vocabulary is cut into: every cluster takes equal jobs in turn, so the shortest end has the fewest rounds times tiles
// a run; a run costs about a tile more than its tiles (its first ones fill the lists), and one state and list a row.  A warp's lanes
// try different numbers; every warp of the launch finds the same.
__device__ __forceinline__ int splits_for(const ScoreParams& p, int row_tiles) {
  const int lane = threadIdx.x & 31, most = min(p.n_tiles, max(1, p.most_jobs / max(1, row_tiles)));
  Key best = ~0ull;
  for (int s = lane + 1; s <= most; s += 32) {
    const unsigned len = (p.n_tiles + s - 1) / s;
    if ((unsigned)s != (p.n_tiles + len - 1) / len) continue;            // the same length with fewer runs
    const Key rounds = ((Key)row_tiles * s + p.clusters - 1) / p.clusters;
    best = min(best, (rounds * (len + 1)) << 20 | (unsigned)s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
  return (int)(best & 0xfffffu);
}

// ------------------------------------------------------------------------------------------------ lists
// A reader thread's list of its row's best classes: `size` entries in shared memory, in no order; entry e of all threads lies together.
struct List {
  float* value;             // this thread's first entry; the next is kReaderThreads further
  int* id;
  int size, used, worst;
  float least;              // a class has to be above it: the worst entry's logit once the list is full
  __device__ __forceinline__ void clear() { used = 0; least = -INFINITY; }
  // Classes come in rising order, so one that equals the worst entry is behind it.
  __device__ __forceinline__ void add(float z, int v) {
    const int at = (used < size ? used : worst) * kReaderThreads;
    value[at] = z;
    id[at] = v;
    used += used < size;
    if (used < size) return;
    worst = 0;
    least = value[0];
#pragma unroll 4
    for (int e = 1; e < size; ++e) {
      const float w = value[e * kReaderThreads];
      if (w < least || (w == least && id[e * kReaderThreads] > id[worst * kReaderThreads])) {
        least = w;
        worst = e;
      }
    }
  }
};

// Adds those of columns v .. v + 15 of a row that belong into its list.  A register cannot be picked by a number, so the columns
// go through shared memory, each thread's own; threads then take theirs at the same time, each its next one.
__device__ __forceinline__ void look_through(const float* x, int v, List& list, float* staging) {
  unsigned found = 0;
#pragma unroll
  for (int i = 0; i < kGroup; ++i) found |= (x[i] > list.least ? 1u : 0u) << i;
  if (!__any_sync(0xffffffffu, found)) return;
#pragma unroll
  for (int i = 0; i < kGroup; ++i) staging[32 * i] = x[i];
  while (__any_sync(0xffffffffu, found)) {
    if (found) {
      const int i = __ffs(found) - 1;
      found &= found - 1;
      const float z = staging[32 * i];
      if (z > list.least) list.add(z, v + i);
    }
  }
}

// ------------------------------------------------------------------------------------------------ product
struct Shared {             // behind the stages, the lists and the staging
  uint64_t full[kMaxStages], empty[kMaxStages];    // a stage holds its operands; the products have read it
  uint64_t acc_full[2], acc_empty[2];              // an accumulator is complete; its readers are done with it
  uint32_t tmem;
  int failed;
  int count[HDET_MAX_REPLICAS];
  int splits;
};

constexpr int kStagingBytes = 4 * kGroup * kReaderThreads;
__host__ __device__ constexpr int list_bytes(int list) { return list ? 8 * list * kReaderThreads + kStagingBytes : 0; }
constexpr int kFixedSmem = 1024 + (int)sizeof(Shared);
static_assert(kFixedSmem + 5 * kStageBytes + list_bytes(kMaxList) <= kMaxSmem, "five stages beside the longest lists");

struct Run {                // a cluster's job: 128 CTAS tokens of a replica, and tiles from .. to of the vocabulary
  int r, m0, from, to;
};

template <int CTAS>
__device__ __forceinline__ bool find_run(const ScoreParams& p, const Shared& sh, int job, Run& run) {
  constexpr int kTile = 128 * CTAS;
  const int splits = sh.splits, len = (p.n_tiles + splits - 1) / splits;
  // tokens fastest: runs that go on at the same time read the same rows of the table
  for (run.r = 0; run.r < p.n_replicas; ++run.r) {
    const int row_tiles = (sh.count[run.r] + kTile - 1) / kTile;
    if (job < row_tiles * splits) {
      run.m0 = job % row_tiles * kTile;
      run.from = job / row_tiles * len;
      run.to = min(run.from + len, p.n_tiles);
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

// 64 columns of a row, from class v on, into its state and list.
template <bool LIST>
__device__ __forceinline__ void take_logits(const ScoreParams& p, float (&x)[2][32], int v, int target, float* z_target, State& s, List& list,
                                            float* staging) {
  cut_columns(x, v, p.vocab);
  const float top = largest(x);
  if ((unsigned)(target - v) < 64u) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (v + i == target) *z_target = x[0][i];
      if (v + 32 + i == target) *z_target = x[1][i];
    }
  }
  if constexpr (LIST) {
    if (__any_sync(0xffffffffu, top > list.least)) {
#pragma unroll
      for (int g = 0; g < 64 / kGroup; ++g) look_through(&x[g / 2][kGroup * (g % 2)], v + kGroup * g, list, staging);
    }
  }
  if (__any_sync(0xffffffffu, top >= s.top && top > -INFINITY)) {
    if (top > s.top) s.raise(top);
    const float m = s.top > -INFINITY ? s.top : NAN;       // equal to nothing
    float n = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const bool is = x[h][i] == m;
        n += is ? 1.0f : 0.0f;
        x[h][i] = is ? -INFINITY : x[h][i];
      }
    s.ties += n;
  }
  const float from = s.top > -INFINITY ? s.top : 0.0f;     // nothing finite yet: exp of -inf, not of NaN
  float e[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float d = x[h][i] - from, y = exp2_fast(d * kLog2e);
      e[i % 4] += y;
      u[i % 4] = fmaf(y, fmaxf(d, -1e4f), u[i % 4]);       // -inf adds 0, not NaN; what is NaN makes e NaN
    }
  s.others += (e[0] + e[1]) + (e[2] + e[3]);
  s.weighted += (u[0] + u[1]) + (u[2] + u[3]);
}

// Tiles of (128 * CTAS) x (128 * CTAS) by a resident CTA (or pair): copies, products and readers each go through the same runs, with a ring
// of stages and two accumulators between them.  Every wait is bounded.
template <int CTAS, bool SUMS, bool LIST>
__global__ void __launch_bounds__(kScoreThreads, 1) scores_kernel(const __grid_constant__ ScoreParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int kTile = 128 * CTAS, kCols = 64 * CTAS;
  const uint32_t smem = (bulk::smem_addr(smem_raw) + 1023u) & ~1023u;
  uint8_t* const behind = smem_raw + (smem - bulk::smem_addr(smem_raw)) + p.stages * kStageBytes;
  Shared& sh = *reinterpret_cast<Shared*>(behind + list_bytes(p.list));
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
    const int splits = splits_for(p, __reduce_add_sync(0xffffffffu, (count + kTile - 1) / kTile));
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
      for (int tile = run.from; go && tile < run.to; ++tile) {
        const int boxes = boxes_for<CTAS>(p.vocab - tile * kTile);
        const int a_row = run.m0 + 128 * (int)rank, b_row = tile * kTile + 64 * boxes * (int)rank;
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
    int s = 0, uses = 0;
    uint32_t parity = 0;
    bool go = true;
    const uint64_t a_desc = operand_desc(smem, kMajor), b_desc = operand_desc(smem + kOperandBytes, kMajor);
    const uint32_t k_step = k_step_bytes(kMajor);
    for (int job = blockIdx.x / CTAS; go && find_run<CTAS>(p, sh, job, run); job += clusters) {
      for (int tile = run.from; go && tile < run.to; ++tile) {
        const uint32_t idesc = instruction_desc<CTAS>(64 * CTAS * boxes_for<CTAS>(p.vocab - tile * kTile), kMajor, kMajor);
        uint32_t acc = 0;
        for (int step = 0, in_chunk = 0; step < steps; ++step) {
          if (in_chunk == 0) {
            const int b = uses & 1;
            if (uses >= 2 && !__all_sync(0xffffffffu, wait_cluster(bar(sh.acc_empty[b]), (uses / 2 - 1) & 1, p.wait_limit))) {
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
          if ((SUMS && in_chunk == p.chunk) || step + 1 == steps) {
            commit<CTAS>(bar(sh.acc_full[uses & 1]));
            ++uses;
            in_chunk = 0;
          }
          if (++s == p.stages) {
            s = 0;
            parity ^= 1;
          }
        }
        if (__any_sync(0xffffffffu, failed)) go = false;
      }
    }
  } else if (warp >= kFirstReader) {
    const int reader = warp - kFirstReader, quarter = warp & 3, half = reader >> 2;
    const int tile_row = 128 * (int)rank + quarter * 32 + lane, thread = 32 * reader + lane;
    List list;
    list.size = p.list;
    list.value = reinterpret_cast<float*>(behind) + thread;
    list.id = reinterpret_cast<int*>(behind + 4 * p.list * kReaderThreads) + thread;
    float* const staging = reinterpret_cast<float*>(behind + 8 * p.list * kReaderThreads) + reader * 32 * kGroup + lane;
    int uses = 0;
    bool go = true;
    for (int job = blockIdx.x / CTAS; go && find_run<CTAS>(p, sh, job, run); job += clusters) {
      const int64_t row = (int64_t)run.r * p.rows_pad + run.m0 + tile_row;
      const int target = p.target[row];
      float* const z_target = p.z_target + row;
      State s;
      s.clear();
      list.clear();
      for (int tile = run.from; go && tile < run.to; ++tile) {
        Columns<SUMS ? CTAS : 0> acc;
        const auto acc_at = [&] { return tmem + (uses & 1) * 128 * CTAS + half * kCols + ((uint32_t)(quarter * 32) << 16); };
        const auto acc_done = [&] {
          fence_before_sync();
          __syncwarp();
          if (lane == 0) arrive_leader(bar(sh.acc_empty[uses & 1]));
          ++uses;
        };
        for (int step = 0; step < steps; step += SUMS ? p.chunk : steps) {
          if (!warp_wait(bar(sh.acc_full[uses & 1]), (uses / 2) & 1, 2 * p.wait_limit)) {
            failed = 1;
            go = false;
            break;
          }
          fence_after_sync();
          if constexpr (SUMS) {
            take_columns(acc_at(), acc, step > 0);
            acc_done();
          }
        }
        if (!go) break;
        Source<CTAS, SUMS> from;
        from.tmem = acc_at();
        from.empty = false;
        if constexpr (SUMS) from.acc = &acc;
#pragma unroll (SUMS ? CTAS : 1)
        for (int c = 0; c < kCols; c += 64) {
          float loaded[2][32];
          float (&x)[2][32] = from.get(c, loaded);
          take_logits<LIST>(p, x, tile * kTile + half * kCols + c, target, z_target, s, list, staging);
        }
        if constexpr (!SUMS) acc_done();
      }
      if (!go) break;
      const int64_t at = ((int64_t)job * 2 + half) * kTile + tile_row;
      p.part[at] = s;
      if constexpr (LIST) {
        Key best = 0;
        Key* to = p.lists + ((int64_t)job * 2 + half) * p.list * kTile + tile_row;
        for (int e = 0; e < p.list; ++e) {
          const Key k = e < list.used ? key_of(list.value[e * kReaderThreads], list.id[e * kReaderThreads]) : 0;
          to[(int64_t)e * kTile] = k;
          best = max(best, k);
        }
        p.best[at] = best;
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
// time, a lane 8 elements of each per step.  A logit is the same in all lanes then, so the warp keeps one state, and its best classes
// in order, one in each lane.
constexpr int kFew = 2, kFewRows = 3;
constexpr int64_t kFewElements = 150000000;      // of all tables, for two tokens: the product is faster beyond

template <int NT>
__global__ void __launch_bounds__(256, 3) few_scores_kernel(const __grid_constant__ ScoreParams p, const __grid_constant__ PackParams k) {
  __shared__ State s_state[8][NT];
  __shared__ Key s_key[NT][8 * 32];
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
  float least[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    s[t].clear();
    mine[t] = 0;
    least[t] = -INFINITY;
  }
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
        s[t].add_logit(z[i][t]);
        if (v + i == target[t] && lane == 0) p.z_target[(int64_t)r * p.rows_pad + t] = z[i][t];
        if (p.list && z[i][t] > least[t]) {
          const Key key = key_of(z[i][t], v + i);
          const int place = __popc(__ballot_sync(0xffffffffu, mine[t] > key));
          const Key above = __shfl_up_sync(0xffffffffu, mine[t], 1);
          mine[t] = lane < place ? mine[t] : lane == place ? key : above;
          const Key last = __shfl_sync(0xffffffffu, mine[t], p.list - 1);
          least[t] = last ? logit_of(last) : -INFINITY;
        }
      }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (lane == 0) s_state[warp][t] = s[t];
    s_key[t][threadIdx.x] = lane < p.list ? mine[t] : 0;
  }
  __syncthreads();
  if (threadIdx.x < count) {
    State all = s_state[0][threadIdx.x];
    for (int i = 1; i < 8; ++i) all.add(s_state[i][threadIdx.x]);
    p.part[((int64_t)r * kFew + threadIdx.x) * p.n_parts + blockIdx.x] = all;
  }
  if (!p.list) return;
  // the block's list: each of the eight lists' entries finds its place by counting those before it
  for (int t = 0; t < count; ++t) {
    const int64_t at = ((int64_t)r * kFew + t) * p.n_parts + blockIdx.x;
    const Key key = s_key[t][threadIdx.x];
    const int held = __syncthreads_count(key != 0);
    int place = 0;
    if (lane < p.list) {
      for (int i = 0; i < 8; ++i)
        for (int e = 0; e < p.list; ++e) place += s_key[t][32 * i + e] > key;
      if (key && place < p.list) {
        p.lists[at * p.list + place] = key;
        if (place == 0) p.best[at] = key;
      }
    }
    if (threadIdx.x >= held && threadIdx.x < p.list) p.lists[at * p.list + threadIdx.x] = 0;
    if (held == 0 && threadIdx.x == 0) p.best[at] = 0;
  }
}

// ------------------------------------------------------------------------------------------------ joining
constexpr int kJoinThreads = 256;
constexpr int kMostParts = 2048;                   // states and lists of a row

// A block a row.  With L lists of C entries each, the row's C best are in the C lists whose first entries are the largest: those are
// found by counting, then the C best of their entries, by counting too.
template <int CTAS>                                // 0: after few_scores_kernel
__global__ void __launch_bounds__(kJoinThreads) join_scores_kernel(const __grid_constant__ ScoreParams p) {
  constexpr int kTile = CTAS ? 128 * CTAS : 1;
  __shared__ State s_state[kJoinThreads / 32];
  __shared__ Key s_first[kMostParts], s_cand[kMaxList * kMaxList], s_best[kMaxList];
  __shared__ double s_exact[kMaxList];
  __shared__ int s_chosen[kMaxList], s_held;
  const int r = blockIdx.y, row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  let_next_start();
  wait_for_previous();
  if (row >= p.count[r]) return;
  // where this row's states and lists are
  int parts = p.n_parts, row_tiles = 0;
  int64_t first_job = 0;
  if constexpr (CTAS) {
    const int splits = p.control->splits;
    for (int i = 0; i < r; ++i) first_job += (p.count[i] + kTile - 1) / kTile;
    first_job = first_job * splits + row / kTile;
    row_tiles = (p.count[r] + kTile - 1) / kTile;
    parts = 2 * splits;
  }
  const auto part_at = [&](int l) -> int64_t {
    if constexpr (CTAS) return ((first_job + (int64_t)(l >> 1) * row_tiles) * 2 + (l & 1)) * kTile + row % kTile;
    else return ((int64_t)r * kFew + row) * p.n_parts + l;
  };
  const auto entry = [&](int l, int e) -> Key {
    if constexpr (CTAS) return p.lists[(((first_job + (int64_t)(l >> 1) * row_tiles) * 2 + (l & 1)) * p.list + e) * kTile + row % kTile];
    else return p.lists[part_at(l) * p.list + e];
  };
  State s;
  s.clear();
  for (int l = threadIdx.x; l < parts; l += kJoinThreads) {
    s.add(p.part[part_at(l)]);
    if (p.list) s_first[l] = p.best[part_at(l)];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s.add_lane(o);
  if (lane == 0) s_state[warp] = s;
  if (threadIdx.x == 0) s_held = 0;
  __syncthreads();
  s = s_state[0];
#pragma unroll
  for (int w = 1; w < kJoinThreads / 32; ++w) s.add(s_state[w]);
  const int64_t at = (int64_t)r * p.rows_pad + row;
  const int token = p.token_of[at];
  // the logarithm of the sum less the maximum's: >= 0
  float rest = logf(s.ties) + log1pf(s.others / s.ties);
  const bool failed = CTAS && p.control->status != 0;
  if (failed || !(fabsf(s.top) < INFINITY) || !(rest < INFINITY)) rest = NAN;
  const ScoreOut& o = p.out;
  if (threadIdx.x == 0) {
    if (o.lse.p) o.lse.at(r, token) = s.top + rest;
    if (o.entropy.p) o.entropy.at(r, token) = rest - s.weighted / (s.ties + s.others);
    if (o.logprob.p) o.logprob.at(r, token) = -((s.top - p.z_target[at]) + rest);
  }
  if (!p.list) return;
  const int list = p.list, n_top = o.n_top;
  if (rest != rest) {
    if (threadIdx.x < n_top) {
      o.top_ids.at(r, (int64_t)token * n_top + threadIdx.x) = -1;
      if (o.top_logprob.p) o.top_logprob.at(r, (int64_t)token * n_top + threadIdx.x) = NAN;
    }
    return;
  }
  int lists = parts;
  if (parts > list) {
    for (int l = threadIdx.x; l < parts; l += kJoinThreads) {
      const Key key = s_first[l];
      int place = 0;
      for (int i = 0; i < parts; ++i) place += s_first[i] > key;
      if (key && place < list) s_chosen[place] = l;
    }
    int some = 0;
    for (int l = threadIdx.x; l < parts; l += kJoinThreads) some += s_first[l] != 0;
    some = __reduce_add_sync(0xffffffffu, some);
    if (lane == 0) atomicAdd(&s_held, some);
    __syncthreads();
    lists = min(list, s_held);
  }
  const int cands = lists * list;
  if (threadIdx.x < list) s_best[threadIdx.x] = 0;
  for (int c = threadIdx.x; c < cands; c += kJoinThreads) s_cand[c] = entry(parts > list ? s_chosen[c / list] : c / list, c % list);
  __syncthreads();
  for (int c = threadIdx.x; c < cands; c += kJoinThreads) {
    const Key key = s_cand[c];
    int place = 0;
    for (int i = 0; i < cands; ++i) place += s_cand[i] > key;
    if (key && place < list) s_best[place] = key;
  }
  __syncthreads();
  // their logits in fp64
  const __nv_bfloat16* h = p.rows + r * p.rows_stride + (p.rows_packed ? row : token) * p.rows_row;
  for (int e = warp; e < list; e += kJoinThreads / 32) {
    const Key key = s_best[e];
    if (!key) continue;
    const __nv_bfloat16* w = p.table + (p.weight_shared ? 0 : r * p.table_stride) + class_of(key) * p.table_row;
    double sum = 0.0;
    if (p.rows_vec) {
      const int whole = p.width & ~7;
      for (int c = lane * 8; c < whole; c += 256) {
        const uint4 a4 = *reinterpret_cast<const uint4*>(h + c), b4 = *reinterpret_cast<const uint4*>(w + c);
        const uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {              // a product of two bf16 numbers is an fp32 number
          sum += (double)(__uint_as_float(a[i] << 16) * __uint_as_float(b[i] << 16));
          sum += (double)(__uint_as_float(a[i] & 0xffff0000u) * __uint_as_float(b[i] & 0xffff0000u));
        }
      }
      if (whole + lane < p.width) sum += (double)(__bfloat162float(h[whole + lane]) * __bfloat162float(w[whole + lane]));
    } else {
      for (int c = lane; c < p.width; c += 32) sum += (double)(__bfloat162float(h[c]) * __bfloat162float(w[c]));
    }
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
    if (lane == 0) s_exact[e] = sum;
  }
  __syncthreads();
  if (threadIdx.x >= list) return;
  const Key key = s_best[threadIdx.x];
  int place = threadIdx.x;                         // of an entry that holds nothing
  if (key) {
    const double z = s_exact[threadIdx.x];
    const int id = class_of(key);
    place = 0;
    for (int i = 0; i < list; ++i) {
      const Key other = s_best[i];
      place += other && (s_exact[i] > z || (s_exact[i] == z && class_of(other) < id));
    }
  }
  if (place < n_top) {
    o.top_ids.at(r, (int64_t)token * n_top + place) = key ? class_of(key) : -1;
    if (o.top_logprob.p) o.top_logprob.at(r, (int64_t)token * n_top + place) = key ? -((s.top - logit_of(key)) + rest) : -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------------ host side
// Whether the table's boxes can be copied from where it is.
bool table_fits(const hdet_token_scores_args* d) {
  return aligned(d->weight, 16) && d->weight_row % 8 == 0 && (d->n_replicas == 1 || d->weight_stride % 8 == 0);
}

constexpr int kSms = 148;        // of a B200, for sizes that must not depend on the device; with another count only times change
constexpr int64_t kFewBlocks = kSms * 3;        // blocks of few_scores_kernel that are resident at once

struct Plan {
  int ctas, tile, list;
  int64_t rows_pad, packed_row, m_tiles, n_tiles;
  bool few, pack_table;
  int64_t n_parts;                // of few_scores_kernel
  int64_t most_jobs;
  int64_t off_count, off_target, off_token, off_z, off_part, off_best, off_lists, off_hidden, off_table, total;
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
  // room for either kernel's: which one runs depends on the hidden states' address, and the size does not
  const int64_t states = std::max<int64_t>(q.most_jobs * 2 * q.tile, T <= kFew ? R * kFew * q.n_parts : 0);
  q.off_part = take(16 * states);
  q.off_best = take(q.list ? 8 * states : 0);
  q.off_lists = take(8 * states * q.list);
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

template <int CTAS, bool SUMS>
auto pick_kernel(bool list) { return list ? scores_kernel<CTAS, SUMS, true> : scores_kernel<CTAS, SUMS, false>; }

cudaError_t prepare(int device, int* sms) {
  const void* kernels[] = {(const void*)scores_kernel<1, false, false>, (const void*)scores_kernel<1, false, true>,
                           (const void*)scores_kernel<1, true, false>,  (const void*)scores_kernel<1, true, true>,
                           (const void*)scores_kernel<2, false, false>, (const void*)scores_kernel<2, false, true>,
                           (const void*)scores_kernel<2, true, false>,  (const void*)scores_kernel<2, true, true>};
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
  p.best = reinterpret_cast<Key*>(ws + q.off_best);
  p.lists = reinterpret_cast<Key*>(ws + q.off_lists);
  p.n_parts = (int)q.n_parts;
  p.n_tiles = (int)q.n_tiles;
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
  const dim3 join_grid((unsigned)d->n_tokens, d->n_replicas);
  if (q.few) {
    p.rows = k.hidden; p.rows_stride = k.hidden_stride; p.rows_row = k.hidden_row;
    p.rows_vec = true;
    const dim3 grid((unsigned)q.n_parts, d->n_replicas);
    e = launch(d->n_tokens == 1 ? few_scores_kernel<1> : few_scores_kernel<2>, grid, 256, 0, 1, st, p, k);
    if (e == cudaSuccess) e = launch(join_scores_kernel<0>, join_grid, kJoinThreads, 0, 1, st, p);
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
  p.clusters = (int)std::min<int64_t>(sms / q.ctas, (int64_t)d->n_replicas * q.m_tiles * q.n_tiles);
  const int lists = list_bytes(q.list);
  p.stages = std::min(kMaxStages, (kMaxSmem - kFixedSmem - lists) / kStageBytes);
  const int smem = kFixedSmem + lists + p.stages * kStageBytes;
  const bool sums = div_up(d->width, kBlockK) > kChunk, list = q.list > 0;
  const auto kernel = q.ctas == 1 ? (sums ? pick_kernel<1, true>(list) : pick_kernel<1, false>(list))
                                  : (sums ? pick_kernel<2, true>(list) : pick_kernel<2, false>(list));
  e = launch(kernel, dim3((unsigned)(p.clusters * q.ctas)), kScoreThreads, smem, q.ctas, st, p);
  if (e == cudaSuccess) e = launch(q.ctas == 1 ? join_scores_kernel<1> : join_scores_kernel<2>, join_grid, kJoinThreads, 0, 1, st, p);
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
