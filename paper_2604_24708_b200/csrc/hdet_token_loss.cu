// Softmax cross entropy of hidden states against a large table, and its gradients, without keeping the logits (contract:
// include/hdet.h).  For each replica, with H the hidden states of its counted tokens, W its table, y the targets:
//
//   Z = H W^T,  lse_t = log sum_v exp Z_tv,  l_t = lse_t - Z_{t,y_t},  loss = mean of l_t
//   P = exp(Z - lse),  G = P - onehot(y),  dH = (c) G W,  dW = (c) G^T H,  c = grad_scale / counted tokens
//
// A likely target's l_t and G are differences of numbers that are nearly equal, so neither is taken as one.  With d = (log of the
// sum of exp over all classes but the target) - Z_{t,y_t}:  l_t = log(1 + exp d)  and  G_{t,y_t} = -1 / (1 + exp -d).
//
// Three products of T x V x D.  G needs lse, which needs all of Z: a piece of the work is as much of G as the workspace holds, as
// many whole replicas as fit, else a part of one replica's vocabulary.
//
//   pack        counted tokens move together (padding drops out: no work, and nothing it holds reaches a product)
// and then, where whole replicas fit and G is bf16, for each group of them
//   numerators  Z tile by tile on the tensor cores; the epilogue keeps, of each half tile's row, its maximum m and the sum of
//               exp(z - m), and leaves exp(z - m) in G's place
//   scale       the row's sum and the token's loss from those; they become G in place; the last block takes the replica's mean
//   grads       both products with G in one launch
// or, forming Z twice (a fourth product, but nothing kept but G),
//   stats       Z, of which the epilogue keeps the maxima and sums
//   join        the row's sum, the token's loss, the replica's mean
// and for each piece of the vocabulary
//   probs       Z again; the epilogue writes G
//   grads       as above; after the last piece, dH's partial sums are joined
// G from given gradients of log probabilities and entropies takes probs' place (given), and then, for rows with one very likely class,
//   likely      that class's entry of G, from the sum of the row's others
// Up to two tokens a replica without gradients take a kernel of their own (few).
//
// G is the operand of a bf16 product, so it is rounded to bf16, unscaled, as the last step of its own.  Its relative error, 2^-8 of a
// value at most, is that of a bf16 gradient's own rounding.  For fp32 gradients that would be too coarse: G is written as the sum of
// three bf16 numbers (24 bits; two would leave up to 2^-16 of a value, 1.3e-6 of a gradient's norm), and the products run over all three.
#include <algorithm>
#include <climits>

#include "hdet_vocab.cuh"

namespace hdet {
namespace {

constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kOperandBytes;
// warp 0 copies, warp 1 issues the products, warp 2 hands out tiles, warps 4 - 11 read the accumulator: a quarter of its
// lanes (warp % 4) and half of its columns each
constexpr int kGemmThreads = 384, kFirstReader = 4, kReaders = 8;
constexpr int kStagingBytes = 4096;        // per reader: 32 rows x 128 bytes
constexpr int kAskAhead = 8;               // steps before a tile's end at which its successor is looked up
constexpr int kTileSlots = 4;              // tiles under way between the copies and the readers
constexpr long long kSelftestLimitCycles = 4000000ll;   // 2 ms

enum Phase { kStats, kNumerators, kProbs, kGrads, kGiven };

struct LossParams {
  CUtensorMap hidden, weight, grad;
  // problem
  int n_replicas, vocab, width, n_tokens;
  int rows_pad;             // rows per replica of everything packed
  bool weight_shared;
  double grad_scale;
  bool of_mean;             // the gradients are those of a mean over the counted tokens
  // packed inputs and per-row values [replica][rows_pad]
  const int* count;
  const int* target;
  const int* token_of;
  float* z_target;
  RowNorm* norm;
  float2* part;             // [replica][rows_pad][n_parts]: Lse of a part of the row
  int n_parts;
  float* row_loss;          // [replica][rows_pad]
  // given gradients (NULL without those of entropies): ScoreGiven's, and sums of the certain rows' entries of G but the likely class's
  const int* certain;
  int* likely;
  float* others;            // [half tile][replica of a launch][rows_pad]
  bool sums_only;           // leaves those sums and nothing of G; `count` is that of the certain rows
  // piece of the vocabulary
  int r0, n_r;              // replicas of this launch
  int v0, v_len, v_pitch;   // first row of the table, rows, pitch of G
  __nv_bfloat16* g;         // [term][replica of a launch][rows_pad][v_pitch]
  int g_terms, g_group;     // terms written; replicas that a term has room for
  // gradients
  int m_tiles, n_tiles;     // stats, probs: tiles of tokens, of the vocabulary
  int h_tiles_m, h_tiles_n, h_splits, h_len, h_jobs;   // dH: tiles, parts of the sum over the vocabulary, 64-steps a part
  int w_tiles_m, w_tiles_n;                            // dW
  int h_terms, w_terms;     // terms of G that each product runs over
  bool h_slabs, h_add;      // dH goes to fp32 partial sums; added to what an earlier piece left
  float* slabs;             // [split][replica of the launch][rows_pad][width]
  Out d_hidden, d_weight;
  float* token_loss;
  int64_t token_loss_stride;
  void* loss;
  int loss_f64;
  Control* control;
  int jobs;                 // tiles of this launch
  int chunk;                // steps of 64 that the tensor core sums before a reader takes them over
  unsigned first_ticket;    // Control::ticket when it starts
  long long wait_limit;     // of every wait, in cycles; twice that where one waits for whole tiles
  bool withhold;            // hands no tile over, so that the waits for it run out (hdet_selftest_token_loss_wait, _token_scores_grad_wait)
};

__device__ __forceinline__ void poison_loss(const LossParams& p) {
  if (!p.loss) return;
  for (int r = 0; r < p.n_replicas; ++r) {
    if (p.loss_f64) static_cast<double*>(p.loss)[r] = NAN; else static_cast<float*>(p.loss)[r] = NAN;
  }
}

// What one CTA (or pair) computes: rows m0.., columns n0.. of a product over k_blocks steps of 64.
struct Job {
  int k_blocks;             // -1: there is none left
  int k_pass;               // steps of one pass over the sum; one pass for each term of a, the smallest first
  int a_pass_z;             // from one term to the next larger one (a_z: the smallest)
  int a_row, a_k, a_z, b_row, b_k, b_z;   // where the operands start
  int r, m0, n0, split;
  int b_boxes;              // boxes of 64 columns that a CTA loads: 2, or 1 where the last tile needs no more
  int is_dw;                // of G^T H; otherwise of G W (kGrads) or H W^T
  int pad;
};
static_assert(sizeof(Job) == 64, "four stores of 16 bytes");

template <int CTAS, int PHASE>
__device__ __forceinline__ bool find_job(const LossParams& p, const int* counts, int tile, Job& j) {
  constexpr int kTile = 128 * CTAS;
  if constexpr (PHASE != kGrads) {
    // tokens fastest: the tiles that run at the same time share rows of the table, and the hidden states stay in L2
    const int per_r = p.m_tiles * p.n_tiles;
    const int g = tile / per_r, rest = tile % per_r;
    j.r = p.r0 + g;
    j.m0 = rest % p.m_tiles * kTile;
    j.n0 = rest / p.m_tiles * kTile;
    if (j.m0 >= counts[j.r]) return false;
    j.a_pass_z = 0;
    j.a_row = j.m0; j.a_k = 0; j.a_z = j.r;
    j.b_row = p.v0 + j.n0; j.b_k = 0; j.b_z = p.weight_shared ? 0 : j.r;
    j.k_pass = j.k_blocks = (p.width + kBlockK - 1) / kBlockK;
    j.split = 0; j.is_dw = 0;
    j.b_boxes = boxes_for<CTAS>(p.v_len - j.n0);
    return true;
  } else {
    // dH first: its sums are the longest, so the short dW tiles fill the machine's end
    if (tile < p.h_jobs) {
      const int per_split = p.n_r * p.h_tiles_m * p.h_tiles_n;
      const int rest = tile % per_split, g = rest / (p.h_tiles_m * p.h_tiles_n), mn = rest % (p.h_tiles_m * p.h_tiles_n);
      j.split = tile / per_split;
      j.r = p.r0 + g;
      j.m0 = mn / p.h_tiles_n * kTile;
      j.n0 = mn % p.h_tiles_n * kTile;
      j.b_boxes = boxes_for<CTAS>(p.width - j.n0);
      if (j.m0 >= counts[j.r]) return false;
      const int all = (p.v_len + kBlockK - 1) / kBlockK;
      const int from = min(j.split * p.h_len, all), to = min(from + p.h_len, all);
      j.k_pass = to - from;
      j.k_blocks = j.k_pass * p.h_terms;
      j.a_pass_z = -p.g_group;
      j.a_row = j.m0; j.a_k = from * kBlockK; j.a_z = g + (p.h_terms - 1) * p.g_group;
      j.b_row = j.n0; j.b_k = p.v0 + from * kBlockK; j.b_z = p.weight_shared ? 0 : j.r;
      j.is_dw = 0;
      return true;
    }
    const int t = tile - p.h_jobs;
    const int g = t / (p.w_tiles_m * p.w_tiles_n), mn = t % (p.w_tiles_m * p.w_tiles_n);
    j.split = 0;
    j.r = p.r0 + g;
    j.m0 = mn / p.w_tiles_n * kTile;
    j.n0 = mn % p.w_tiles_n * kTile;
    j.b_boxes = boxes_for<CTAS>(p.width - j.n0);
    j.k_pass = (counts[j.r] + kBlockK - 1) / kBlockK;
    j.k_blocks = j.k_pass * p.w_terms;
    j.a_pass_z = -p.g_group;
    j.a_row = j.m0; j.a_k = 0; j.a_z = g + (p.w_terms - 1) * p.g_group;
    j.b_row = j.n0; j.b_k = 0; j.b_z = j.r;
    j.is_dw = 1;
    return true;
  }
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Numerators, 0 <= x <= 1, in 16 bits: ten bits of mantissa, six of exponent, no sign: the middle bits of x / 2^64 as fp32.  Off by
// 2^-11 of the value down to 2^-62, an eighth of the rounding of G to bf16 that follows; zero below.  (fp16, used before, is off by
// more than that rounding below 2^-16 of the row's largest neighbour and zero below 2^-25: gradients of unlikely classes were lost.)
constexpr float kNumeratorBits = 64.0f, kNumeratorUnit = 18446744073709551616.0f;   // 2^64

// Two values x / 2^64.
__device__ __forceinline__ uint32_t numerator_pair(float lo, float hi) {
  return __byte_perm((__float_as_uint(lo) + 0x1000u) << 3, (__float_as_uint(hi) + 0x1000u) << 3, 0x7632);
}

__device__ __forceinline__ float2 numerators_of(uint32_t pair) {
  return make_float2(__uint_as_float((pair & 0xffffu) << 13), __uint_as_float(pair >> 16 << 13));
}

// ------------------------------------------------------------------------------------------------ epilogues
// Staged rows of 32 fp32 values, columns col .., added to (or put in the place of) what a gradient holds.
__device__ __forceinline__ void add_staged(const Rows& rows, uint32_t at, int lane, int col, int width, bool f32, bool accumulate) {
  __syncwarp();
  const int chunk = lane & 7, c = col + 4 * chunk;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 4 * i + (lane >> 3);
    const uint4 u = unstage(at, row, chunk);
    float4 v = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
    const int64_t offset = __shfl_sync(0xffffffffu, rows.offset, row);
    if (!(rows.on >> row & 1) || c >= width) continue;
    char* row_at = rows.base + offset;
    if (f32) {
      float4* to = reinterpret_cast<float4*>(row_at + 4 * (int64_t)c);
      if (accumulate) {
        const float4 old = *to;
        v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
      }
      *to = v;
    } else {
      uint2* to = reinterpret_cast<uint2*>(row_at + 2 * (int64_t)c);
      if (accumulate) {
        const uint2 old = *to;
        v.x += __uint_as_float(old.x << 16); v.y += __uint_as_float(old.x & 0xffff0000u);
        v.z += __uint_as_float(old.y << 16); v.w += __uint_as_float(old.y & 0xffff0000u);
      }
      *to = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
    }
  }
  __syncwarp();
}

// The same for gradients whose rows do not start and end on 16-byte boundaries: a row's 32 values by 32 threads (13 x 3383 tokens x
// 138, width 763, bf16: 379 us for the call; 586 when each thread wrote its own row's).
__device__ __forceinline__ void write_elements(const Rows& rows, uint32_t at, int lane, int col, int width, bool f32, bool accumulate) {
  __syncwarp();
  const int c = col + lane;
#pragma unroll 4
  for (int row = 0; row < 32; ++row) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4) : "memory");
    const int64_t offset = __shfl_sync(0xffffffffu, rows.offset, row);
    if (!(rows.on >> row & 1) || c >= width) continue;
    if (f32) {
      float* to = reinterpret_cast<float*>(rows.base + offset) + c;
      *to = accumulate ? *to + v : v;
    } else {
      __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(rows.base + offset) + c;
      *to = __float2bfloat16_rn(accumulate ? __bfloat162float(*to) + v : v);
    }
  }
  __syncwarp();
}

// A sum of exponentials, sum * exp(top); top = -inf: of nothing.
struct Lse {
  float top, sum;
  __device__ __forceinline__ void add(float2 o) {
    const float now = fmaxf(top, o.x);
    const float from = now == -INFINITY ? 0.0f : now;
    sum = sum * exp_from(top, from) + o.y * exp_from(o.x, from);
    top = now;
  }
  __device__ __forceinline__ void add_logit(float z) { add(make_float2(z, 1.0f)); }
  __device__ __forceinline__ void add_warp() {     // over a warp's lanes, in a fixed order
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) add(make_float2(__shfl_xor_sync(0xffffffffu, top, o), __shfl_xor_sync(0xffffffffu, sum, o)));
  }
};

// `others`: a row's classes but its target; `z`: the target's logit.
struct Target {
  float loss, grad;         // its loss, and its entry of G
  __device__ __forceinline__ Target(const Lse& others, float z) {
    float d = (others.top - z) + logf(others.sum);
    if (z == INFINITY) d = NAN;                    // as inf - inf
    const float e = expf(-fabsf(d));
    loss = fmaxf(d, 0.0f) + log1pf(e);
    grad = d < 0.0f ? -e / (1.0f + e) : -1.0f / (1.0f + e);
  }
};

__device__ __forceinline__ RowNorm norm_of(const Lse& others, float z, float grad) {
  const float top = others.top == -INFINITY ? z : others.top;
  return RowNorm{top, 1.0f / (others.sum + exp_from(z, top)), grad, 0.0f};
}

// Takes the target's logit out, -inf in its place.
__device__ __forceinline__ void take_target(float (&x)[2][32], int v, int target, float& taken) {
  if ((unsigned)(target - v) >= 64u) return;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (v + i == target) { taken = x[0][i]; x[0][i] = -INFINITY; }
    if (v + 32 + i == target) { taken = x[1][i]; x[1][i] = -INFINITY; }
  }
}

// exp(x - top) 2^shift in place; returns the sum.
__device__ __forceinline__ float exponentials(float (&x)[2][32], float top, float shift = 0.0f) {
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    x[0][i] = exp_from(x[0][i], top, shift); x[0][i + 1] = exp_from(x[0][i + 1], top, shift);
    x[1][i] = exp_from(x[1][i], top, shift); x[1][i + 1] = exp_from(x[1][i + 1], top, shift);
    s[0] += x[0][i]; s[1] += x[0][i + 1]; s[2] += x[1][i]; s[3] += x[1][i + 1];
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// `from`: the reader's row, its half of the tile's columns; `half`: the first of those within the tile.
template <int CTAS, bool SUMS>
__device__ __forceinline__ void stats_epilogue(const LossParams& p, const Job& j, const Source<CTAS, SUMS>& from, int row, int half, int target) {
  constexpr int kCols = 64 * CTAS;
  const int64_t at = (int64_t)j.r * p.rows_pad + row;
  const int v0 = j.n0 + half;
  Lse l{-INFINITY, 0.0f};
  float taken = 0.0f;
#pragma unroll (SUMS ? CTAS : 1)
  for (int c = 0; c < kCols; c += 64) {
    float loaded[2][32];
    float (&x)[2][32] = from.get(c, loaded);
    cut_columns(x, v0 + c, p.vocab);
    take_target(x, v0 + c, target, taken);
    const float top = largest(x);
    const float s = exponentials(x, top == -INFINITY ? 0.0f : top);    // nothing finite: exp of -inf, not of NaN
    l.add(make_float2(top, s));
  }
  p.part[at * p.n_parts + v0 / kCols] = make_float2(l.top, l.sum);
  if (target >= v0 && target < v0 + kCols) p.z_target[at] = taken;
}

// The same, and the numerators exp(z - maximum of the half tile's row) go to the workspace, where scale_kernel turns them
// into G.  The sum is taken before they are rounded.
template <int CTAS, bool SUMS>
__device__ __forceinline__ void numerators_epilogue(const LossParams& p, const Job& j, const Source<CTAS, SUMS>& from, int row, int half,
                                                    int target, uint32_t staging, int lane) {
  constexpr int kCols = 64 * CTAS;
  const int64_t at = (int64_t)j.r * p.rows_pad + row;
  const int v0 = j.n0 + half;
  float top = -INFINITY, sum = 0.0f, taken = 0.0f;
#pragma unroll (SUMS ? CTAS : 1)
  for (int c = 0; c < kCols; c += 64) {
    float loaded[2][32];
    float (&x)[2][32] = from.get(c, loaded);
    cut_columns(x, v0 + c, p.vocab);
    take_target(x, v0 + c, target, taken);
    top = fmaxf(top, largest(x));
  }
  const float from_top = top == -INFINITY ? 0.0f : top;
  Rows rows;
  rows.base = reinterpret_cast<char*>(p.g);
  rows.offset = (((int64_t)(j.r - p.r0) * p.rows_pad + row) * p.v_pitch + v0) * 2;
  rows.on = 0xffffffffu;
#pragma unroll (SUMS ? CTAS : 1)
  for (int c = 0; c < kCols; c += 64) {
    float loaded[2][32];
    float (&x)[2][32] = from.get(c, loaded);
    cut_columns(x, v0 + c, p.vocab);
    float again;
    take_target(x, v0 + c, target, again);
    sum += exponentials(x, from_top, -kNumeratorBits);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* y = &x[i / 4][8 * (i % 4)];
      stage(staging, lane, i, make_uint4(numerator_pair(y[0], y[1]), numerator_pair(y[2], y[3]), numerator_pair(y[4], y[5]),
                                              numerator_pair(y[6], y[7])));
    }
    write_staged(rows, staging, lane, 2 * c, 2 * kCols);
  }
  p.part[at * p.n_parts + v0 / kCols] = make_float2(top, sum * kNumeratorUnit);
  if (target >= v0 && target < v0 + kCols) p.z_target[at] = taken;
}

// kGiven: G from given gradients of log probabilities and entropies in place of the loss's.  CERTAIN: of the first `certain` rows the likely
// class's entry is 0 for now, and the others are summed (in memory beyond 64 of them: a register that lasts is one that the kernel does not have).
template <int CTAS, int PHASE, bool SUMS, bool CERTAIN>
__device__ __forceinline__ void probs_epilogue(const LossParams& p, const Job& j, const Source<CTAS, SUMS>& from, int row, int half, bool counted,
                                               int certain, int target, const RowNorm& norm, uint32_t staging, int lane) {
  constexpr int kCols = 64 * CTAS;
  target = counted ? target - p.v0 : -1;
  const int v0 = j.n0 + half;
  const bool some = CERTAIN && __any_sync(0xffffffffu, row < certain);
  Rows rows;
  rows.offset = (((int64_t)(j.r - p.r0) * p.rows_pad + row) * p.v_pitch + v0) * 2;
  rows.on = 0xffffffffu;
#pragma unroll (SUMS ? CTAS : 1)
  for (int c = 0; c < kCols; c += 64) {
    float loaded[2][32];
    float (&x)[2][32] = from.get(c, loaded);
    if (some && row < certain && largest(x) - norm.top > kLikely) {
#pragma unroll
      for (int i = 0; i < 64; ++i)
        if (v0 + c + i < p.v_len && x[i / 32][i % 32] - norm.top > kLikely) {
          p.likely[(int64_t)j.r * p.rows_pad + row] = p.v0 + v0 + c + i;
          x[i / 32][i % 32] = -INFINITY;
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int v = v0 + c + 32 * h;
      if constexpr (PHASE == kGiven) {             // two columns an instruction where there is one for it
        const uint64_t top = pair_of(-norm.top, -norm.top), scale = pair_of(kLog2e, kLog2e);
        const uint64_t slope = pair_of(-norm.slope, -norm.slope), inverse = pair_of(-norm.inverse, -norm.inverse);
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          const uint64_t d = add_pair(pair_of(x[h][i], x[h][i + 1]), top);
          float a, b;
          halves_of(mul_pair(d, scale), a, b);
          a = exp2_fast(a);
          b = exp2_fast(b);
          // a logit of -inf: 0, not NaN; one that is NaN stays so
          float f, g;
          halves_of(d, f, g);
          halves_of(mul_pair(pair_of(a, b), fma_pair(slope, pair_of(fmaxf(f, -1e4f), fmaxf(g, -1e4f)), inverse)), x[h][i], x[h][i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) x[h][i] = exp_from(x[h][i], norm.top) * norm.inverse;
      }
      if ((unsigned)(target - v) < 32u) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (v + i == target) x[h][i] = norm.target;
      }
      if (!counted || v + 32 > p.v_len) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (!counted || v + i >= p.v_len) x[h][i] = 0.0f;
      }
    }
    if (some) {
      uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 64; i += 2) sum[i / 2 % 4] = add_pair(sum[i / 2 % 4], pair_of(x[i / 32][i % 32], x[i / 32][i % 32 + 1]));
      float a, b;
      halves_of(add_pair(add_pair(sum[0], sum[1]), add_pair(sum[2], sum[3])), a, b);
      if (row < certain) {
        float* to = p.others + ((int64_t)((p.v0 + v0) / kCols) * p.g_group + (j.r - p.r0)) * p.rows_pad + row;
        *to = c ? *to + (a + b) : a + b;
      }
    }
    if (CERTAIN && p.sums_only) continue;
    // each term goes out, and what it leaves of each value stays in its place for the next
    for (int term = 0; term < p.g_terms; ++term) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float* y = &x[k / 4][8 * (k % 4)];
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = bf16_pair(y[2 * i], y[2 * i + 1]);
          y[2 * i] -= __uint_as_float(w[i] << 16);
          y[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
        }
        stage(staging, lane, k, make_uint4(w[0], w[1], w[2], w[3]));
      }
      rows.base = reinterpret_cast<char*>(p.g + (int64_t)term * p.g_group * p.rows_pad * p.v_pitch);
      write_staged(rows, staging, lane, 2 * c, 2 * kCols);
    }
  }
}

template <int CTAS, bool SUMS>
__device__ __forceinline__ void grads_epilogue(const LossParams& p, const Job& j, const Source<CTAS, SUMS>& from, int row, int half, int count,
                                               uint32_t staging, int lane) {
  constexpr int kCols = 64 * CTAS;
  Out o;
  int64_t base;
  float scale = (float)(p.grad_scale / (double)(p.of_mean && count > 0 ? count : 1));
  bool on;
  if (j.is_dw) {
    o = p.d_weight;
    on = row < p.v_len;
    base = j.r * o.stride + (int64_t)(p.v0 + row) * o.row;
  } else if (p.h_slabs) {
    o.p = p.slabs; o.f32 = 1; o.accumulate = p.h_add; o.vec = p.width % 4 == 0;
    on = row < count;
    base = (((int64_t)j.split * p.n_r + (j.r - p.r0)) * p.rows_pad + row) * p.width;
    scale = 1.0f;
  } else {
    o = p.d_hidden;
    on = row < count;
    base = on ? j.r * o.stride + (int64_t)p.token_of[(int64_t)j.r * p.rows_pad + row] * o.row : 0;
  }
  const int n0 = j.n0 + half;
  Rows rows;
  rows.base = static_cast<char*>(o.p);
  rows.offset = base * (o.f32 ? 4 : 2);
  rows.on = __ballot_sync(0xffffffffu, on);
#pragma unroll (SUMS ? CTAS : 1)
  for (int c = 0; c < kCols; c += 64) {
    if (n0 + c >= p.width) break;
    float loaded[2][32];
    float (&x)[2][32] = from.get(c, loaded);
#pragma unroll
    for (int i = 0; i < 32; ++i) { x[0][i] *= scale; x[1][i] *= scale; }
    if (o.vec && !o.f32 && !o.accumulate) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* y = &x[k / 4][8 * (k % 4)];
        stage(staging, lane, k, make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])));
      }
      write_staged(rows, staging, lane, 2 * (int64_t)(n0 + c), 2 * (int64_t)p.width);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          stage(staging, lane, k, make_uint4(__float_as_uint(x[h][4 * k]), __float_as_uint(x[h][4 * k + 1]),
                                             __float_as_uint(x[h][4 * k + 2]), __float_as_uint(x[h][4 * k + 3])));
        if (o.vec) add_staged(rows, staging, lane, n0 + c + 32 * h, p.width, o.f32, o.accumulate);
        else write_elements(rows, staging, lane, n0 + c + 32 * h, p.width, o.f32, o.accumulate);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ product
struct Shared {             // behind the stages and the readers' staging
  uint64_t full[kStages], empty[kStages];          // a stage holds its operands; the products have read it
  uint64_t acc_full[2], acc_empty[2];              // an accumulator is complete; its readers are done with it
  uint64_t tile_full[kTileSlots], tile_empty[kTileSlots], taken;   // taken: the leader's copies have the last tile published
  alignas(16) Job job[kTileSlots];
  uint32_t tmem;
  int failed;
  int count[HDET_MAX_REPLICAS], certain[HDET_MAX_REPLICAS];
};

constexpr int kGemmSmem = 1024 + kStages * kStageBytes + kReaders * kStagingBytes + (int)sizeof(Shared);
static_assert(kGemmSmem <= 227 * 1024, "shared memory of one CTA");

// Tiles of (128 * CTAS) x (128 * CTAS), one CTA a SM (a pair for each two) that stays: the copies run ahead into the next
// tile while the products finish this one, and two accumulators let the readers empty one while the other fills.  Tiles
// differ in length (a replica's counted tokens, dH beside dW), so they are handed out one by one: a thread of the leader draws
// the next number, works out what it means and gives that to both CTAs, a tile ahead (worked out where it is used,
// with its divisions, it held up the copies at every tile: 1.38 ms became 1.51 for 8 x 2048 tokens of width 1024).  The
// counter goes on from launch to launch of a call; every launch draws `jobs` numbers (each cluster's first tile needs none, its
// last number is one too many), so the host knows where the next begins.
//
// The tensor cores do not round the sums they keep, they cut them: an error of up to a step of fp32 towards zero for every 16
// products, which adds up.  A table of 50257 rows makes 6284 times of it, and dH in fp32 was 9.6e-5 off.  So the sum is
// taken out every `chunk` steps and goes on in the readers' registers, in fp32 and rounded, while the other accumulator
// fills.
template <int CTAS, int PHASE, bool SUMS>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_kernel(const __grid_constant__ LossParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem = (bulk::smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t staging0 = smem + kStages * kStageBytes;
  Shared& sh = *reinterpret_cast<Shared*>(smem_raw + (staging0 - bulk::smem_addr(smem_raw)) + kReaders * kStagingBytes);
  volatile int& failed = sh.failed;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 1 ? 0 : cluster_rank();
  const auto bar = [](const uint64_t& b) { return bulk::smem_addr(&b); };

  let_next_start();
  if (threadIdx.x == 96) {                       // a warp that has nothing else to do
    prefetch_map(&p.weight);
    prefetch_map(&p.hidden);
    if constexpr (PHASE == kGrads) prefetch_map(&p.grad);
  }
  if (threadIdx.x == 0) {
    sh.failed = 0;
    for (int s = 0; s < kStages; ++s) {
      bulk::barrier_init(bar(sh.full[s]), 1);
      bulk::barrier_init(bar(sh.empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      bulk::barrier_init(bar(sh.acc_full[b]), 1);
      bulk::barrier_init(bar(sh.acc_empty[b]), kReaders * CTAS);
    }
    for (int q = 0; q < kTileSlots; ++q) {
      bulk::barrier_init(bar(sh.tile_full[q]), 1);
      bulk::barrier_init(bar(sh.tile_empty[q]), (1 + kReaders) * CTAS + 1);   // copies and readers, and the leader's products
    }
    bulk::barrier_init(bar(sh.taken), 1);
    bulk::barrier_init_fence();
  }
  if (warp == 1) tmem_alloc<CTAS>(bulk::smem_addr(&sh.tmem), 2 * 128 * CTAS);
  wait_for_previous();
  if (threadIdx.x < p.n_replicas) {
    sh.count[threadIdx.x] = p.count[threadIdx.x];
    if constexpr (PHASE == kGiven) sh.certain[threadIdx.x] = p.certain ? p.certain[threadIdx.x] : 0;
  }
  fence_before_sync();
  __syncthreads();
  if constexpr (CTAS == 2) cluster_sync();       // the peer's barriers exist before anything arrives there
  fence_after_sync();
  const uint32_t tmem = sh.tmem;

  const auto arrive_leader = [&](uint32_t at) {
    if (rank == 0) bulk::barrier_arrive(at); else arrive_cluster(in_cta(at, 0));
  };
  // The i-th tile of this cluster (the first is its own, the others are handed out); false when there is none left, or a
  // wait ran out.
  const auto next_job = [&](int i, Job& j) -> bool {
    if (i == 0) {
      if (!find_job<CTAS, PHASE>(p, sh.count, blockIdx.x / CTAS, j)) j.k_blocks = -2;   // nothing counted there
      return true;
    }
    const int use = i - 1, q = use % kTileSlots;
    const bool ok = wait_cluster(bar(sh.tile_full[q]), (use / kTileSlots) & 1, 2 * p.wait_limit);
    if (!__all_sync(0xffffffffu, ok)) {
      failed = 1;
      return false;
    }
    const uint32_t from = bulk::smem_addr(&sh.job[q]);
    int* to = reinterpret_cast<int*>(&j);
#pragma unroll
    for (int k = 0; k < 16; k += 4)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(to[k]), "=r"(to[k + 1]), "=r"(to[k + 2]), "=r"(to[k + 3])
                   : "r"(from + 4 * k)
                   : "memory");
    // one value for the warp, so that what is worked out from it is the warp's too
#pragma unroll
    for (int k = 0; k < 15; ++k) to[k] = __shfl_sync(0xffffffffu, to[k], 0);
    if (lane == 0) {
      arrive_leader(bar(sh.tile_empty[q]));
      if (warp == 0 && rank == 0) bulk::barrier_arrive(bar(sh.taken));
    }
    return j.k_blocks >= 0 && __all_sync(0xffffffffu, !failed);
  };
  // operands of this kernel's products: G W, G^T H, or H W^T
  const auto a_mn = [&](const Job& j) { return PHASE == kGrads && j.is_dw; };
  constexpr bool b_mn = PHASE == kGrads;

  // no row is certain: the launch hands its numbers back, and nothing waits
  bool idle = PHASE == kGiven && p.sums_only;
  if constexpr (PHASE == kGiven) {
    if (idle)
      for (int r = 0; r < p.n_r; ++r) idle = idle && sh.certain[p.r0 + r] == 0;
  }
  if (idle) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicAdd(&p.control->ticket, (unsigned)p.jobs);
  } else if (warp == 0) {
    {
      int kb = 0, s = 0;                         // stages filled so far, the next stage
      uint32_t parity = 0;                       // of the ring's present round
      const CUtensorMap* const a_map = PHASE == kGrads ? &p.grad : &p.hidden;
      Job j, next;
      bool more = next_job(0, j);
      for (int i = 0; more; ++i, j = next) {
        const int ask_at = j.k_blocks > kAskAhead ? j.k_blocks - kAskAhead : 0;   // the next tile is looked up while this one is under way
        const CUtensorMap* const b_map = j.is_dw ? &p.hidden : &p.weight;
        const bool a_outer = a_mn(j);
        const int a_row = j.a_row + 128 * (int)rank, b_row = j.b_row + 64 * j.b_boxes * (int)rank;
        int in_pass = 0, a_z = j.a_z;
        for (int step = 0; step < j.k_blocks; ++step, ++kb) {
          if (kb >= kStages && !warp_wait(bar(sh.empty[s]), parity ^ 1, p.wait_limit)) {
            failed = 1;
            break;
          }
          const uint32_t full = bar(sh.full[s]);
          if (rank == 0) expect_bytes(full, CTAS * (kOperandBytes + j.b_boxes * kBoxBytes));
          const uint32_t done = CTAS == 1 ? full : in_cta(full, 0);
          const uint32_t dst = smem + s * kStageBytes;
          if (in_pass == j.k_pass) {
            in_pass = 0;
            a_z += j.a_pass_z;
          }
          const int k = in_pass++ * kBlockK;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (a_outer) load_box<CTAS>(dst + h * kBoxBytes, a_map, a_row + 64 * h, j.a_k + k, a_z, done);
            else load_box<CTAS>(dst + h * kBoxBytes, a_map, j.a_k + k, a_row + 64 * h, a_z, done);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h >= j.b_boxes) break;
            if (b_mn) load_box<CTAS>(dst + kOperandBytes + h * kBoxBytes, b_map, b_row + 64 * h, j.b_k + k, j.b_z, done);
            else load_box<CTAS>(dst + kOperandBytes + h * kBoxBytes, b_map, j.b_k + k, b_row + 64 * h, j.b_z, done);
          }
          if (++s == kStages) {
            s = 0;
            parity ^= 1;
          }
          if (step == ask_at) more = next_job(i + 1, next);
        }
        if (j.k_blocks <= 0) more = next_job(i + 1, next);
        if (__any_sync(0xffffffffu, failed)) break;
      }
      // the products have read the last stages: every arrival that was sent to this CTA's barriers is in
      for (int k = kb > kStages ? kb - kStages : 0; k < kb && __all_sync(0xffffffffu, !failed); ++k)
        if (!warp_wait(bar(sh.empty[k % kStages]), (k / kStages) & 1, p.wait_limit)) failed = 1;
    }
  } else if (warp == 1) {
    if (rank == 0) {
      int s = 0, uses = 0;
      uint32_t parity = 0;
      Job j, next;
      bool more = next_job(0, j);
      for (int i = 0; more; ++i, j = next) {
        const int ask_at = j.k_blocks > kAskAhead ? j.k_blocks - kAskAhead : 0;
        const uint32_t idesc = instruction_desc<CTAS>(64 * CTAS * j.b_boxes, a_mn(j), b_mn);
        const uint32_t a_step = k_step_bytes(a_mn(j)), b_step = k_step_bytes(b_mn);
        const uint64_t a_desc = operand_desc(smem, a_mn(j)), b_desc = operand_desc(smem + kOperandBytes, b_mn);
        uint32_t acc = 0;
        for (int step = 0, in_chunk = 0; step < j.k_blocks; ++step) {
          if (in_chunk == 0) {
            const int b = uses & 1;
            if (uses >= 2 && !__all_sync(0xffffffffu, wait_cluster(bar(sh.acc_empty[b]), (uses / 2 - 1) & 1, p.wait_limit))) {
              failed = 1;
              break;
            }
            fence_after_sync();
            acc = tmem + b * 128 * CTAS;
          }
          if (!warp_wait(bar(sh.full[s]), parity, p.wait_limit)) {
            failed = 1;
            break;
          }
          fence_after_sync();
#pragma unroll
          for (int k = 0; k < kBlockK / 16; ++k)   // addresses are the descriptors' low bits, in units of 16 bytes
            mma<CTAS>(acc, a_desc + (uint32_t)(s * kStageBytes + k * a_step) / 16, b_desc + (uint32_t)(s * kStageBytes + k * b_step) / 16, idesc,
                      in_chunk > 0 || k > 0);
          commit<CTAS>(bar(sh.empty[s]));
          ++in_chunk;
          if ((SUMS && in_chunk == p.chunk) || step + 1 == j.k_blocks) {
            commit<CTAS>(bar(sh.acc_full[uses & 1]));
            ++uses;
            in_chunk = 0;
          }
          if (++s == kStages) {
            s = 0;
            parity ^= 1;
          }
          if (step == ask_at) more = next_job(i + 1, next);
        }
        if (j.k_blocks <= 0) more = next_job(i + 1, next);
        if (__any_sync(0xffffffffu, failed)) break;
      }
    }
  } else if (warp == 2) {
    if (lane == 0 && rank == 0 && !p.withhold) {
      const unsigned clusters = gridDim.x / CTAS;
      // A number is drawn when the copies have taken the one before: one drawn earlier may be a tile that another cluster, with
      // nothing left to do, could have had (four drawn ahead: 102 us instead of 77 for 3 x 129 tokens x 4099, width 520).
      for (int use = 0;;) {
        const int q = use % kTileSlots;
        if ((use > 0 && !bulk::barrier_wait(bar(sh.taken), (use - 1) & 1, 2 * p.wait_limit)) ||
            (use >= kTileSlots && !wait_cluster(bar(sh.tile_empty[q]), (use / kTileSlots - 1) & 1, 2 * p.wait_limit))) {
          failed = 1;
          break;
        }
        const unsigned t = atomicAdd(&p.control->ticket, 1u) - p.first_ticket;
        const bool last = t >= (unsigned)p.jobs - clusters;
        Job j;
        if (!last && !find_job<CTAS, PHASE>(p, sh.count, (int)(t + clusters), j)) continue;   // nothing counted there
        if (last) j.k_blocks = -1;
        ++use;
        const int* from = reinterpret_cast<const int*>(&j);
#pragma unroll
        for (int c = 0; c < CTAS; ++c) {
          const uint32_t to = in_cta(bulk::smem_addr(&sh.job[q]), c);
#pragma unroll
          for (int k = 0; k < 16; ++k) store_cluster(to + 4 * k, from[k]);
          arrive_cluster(in_cta(bar(sh.tile_full[q]), c));
        }
        if (last) break;
      }
    }
  } else if (warp >= kFirstReader) {
    const int reader = warp - kFirstReader, quarter = warp & 3, half = (reader >> 2) * 64 * CTAS;
    const uint32_t staging = staging0 + reader * kStagingBytes;
    int uses = 0;
    Job j;
    for (int i = 0; next_job(i, j); ++i) {
      if (j.k_blocks < 0) continue;                // the cluster's first, with nothing counted
      const int row = j.m0 + 128 * (int)rank + quarter * 32 + lane;
      int target = -1;                             // -1 behind the counted tokens, too
      RowNorm norm{INFINITY, 0.0f, 0.0f, 0.0f};
      if constexpr (PHASE != kGrads) {
        target = p.target[(int64_t)j.r * p.rows_pad + row];
        if ((PHASE == kProbs || PHASE == kGiven) && row < sh.count[j.r]) norm = p.norm[(int64_t)j.r * p.rows_pad + row];
      }
      Columns<SUMS ? CTAS : 0> acc;
      if constexpr (SUMS) {
        if (j.k_blocks == 0) clear(acc);
      }
      const auto acc_at = [&] { return tmem + (uses & 1) * 128 * CTAS + half + ((uint32_t)(quarter * 32) << 16); };
      const auto acc_done = [&] {
        fence_before_sync();
        __syncwarp();
        if (lane == 0) arrive_leader(bar(sh.acc_empty[uses & 1]));
        ++uses;
      };
      bool ok = true;
      for (int step = 0; step < j.k_blocks; step += SUMS ? p.chunk : j.k_blocks) {
        ok = warp_wait(bar(sh.acc_full[uses & 1]), (uses / 2) & 1, 2 * p.wait_limit);
        if (!ok) break;
        fence_after_sync();
        if constexpr (SUMS) {
          take_columns(acc_at(), acc, step > 0);
          acc_done();
        }
      }
      if (!ok) {
        failed = 1;
        break;
      }
      Source<CTAS, SUMS> from;
      from.tmem = acc_at();
      from.empty = j.k_blocks == 0;
      if constexpr (SUMS) from.acc = &acc;
      if constexpr (PHASE == kStats) stats_epilogue(p, j, from, row, half, target);
      else if constexpr (PHASE == kNumerators) numerators_epilogue(p, j, from, row, half, target, staging, lane);
      else if constexpr (PHASE == kProbs || PHASE == kGiven) {
        // Two forms, since the second's few branches make the first 6 % longer; in the second's place alone where sums leave no registers for both
        // (1232 bytes spilled).
        if (PHASE == kGiven && (SUMS || __any_sync(0xffffffffu, row < sh.certain[j.r])))
          probs_epilogue<CTAS, PHASE, SUMS, PHASE == kGiven>(p, j, from, row, half, row < sh.count[j.r], sh.certain[j.r], target, norm, staging, lane);
        else
          probs_epilogue<CTAS, PHASE, SUMS, false>(p, j, from, row, half, row < sh.count[j.r], 0, target, norm, staging, lane);
      } else grads_epilogue(p, j, from, row, half, sh.count[j.r], staging, lane);
      if constexpr (!SUMS) {
        if (j.k_blocks > 0) acc_done();
      }
    }
  }
  __syncwarp();
  fence_before_sync();
  __syncthreads();
  if (sh.failed && threadIdx.x == 0) {
    atomicExch(&p.control->status, 1u);
    poison_loss(p);
    // Copies into this CTA's shared memory and products that read it may still be under way; after this they are not.  A wait on their
    // barriers would not see all of them: a pair's second CTA may have issued copies that the first, whose barriers count them, has not
    // announced.
    for (const long long start = clock64(); clock64() - start < kDrainCycles;) __nanosleep(1000);
  }
  if constexpr (CTAS == 2) cluster_sync();       // neither CTA leaves while the other may still reach into it
  fence_after_sync();
  if (warp == 1) tmem_free<CTAS>(tmem, 2 * 128 * CTAS);
}

// ------------------------------------------------------------------------------------------------ joining
// A row's loss, where it belongs.
__device__ __forceinline__ void write_row(const LossParams& p, int r, int row, float loss, int token) {
  p.row_loss[(int64_t)r * p.rows_pad + row] = loss;
  if (p.token_loss) p.token_loss[r * p.token_loss_stride + token] = loss;
}

// After a block has written its rows' losses: the last of a replica's `blocks` adds them up (fp64, in a fixed order) and
// writes the mean.  256 threads.
__device__ __forceinline__ void finish_block(const LossParams& p, int r, unsigned blocks) {
  __shared__ bool s_last;
  __shared__ double s_sum[8];
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(&p.control->done[r], 1u) == blocks - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  const int count = p.count[r];
  double sum = 0.0;
  for (int row = threadIdx.x; row < count; row += 256) sum += (double)__ldcg(p.row_loss + (int64_t)r * p.rows_pad + row);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 8; ++w) sum += s_sum[w];
  double mean = count > 0 ? sum / (double)count : 0.0;
  if (__ldcg(&p.control->status)) mean = NAN;
  if (p.loss_f64) static_cast<double*>(p.loss)[r] = mean; else static_cast<float*>(p.loss)[r] = (float)mean;
}

// Sum and loss of a row from its parts, one warp a row.
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ LossParams p) {
  const int r = blockIdx.y, row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  let_next_start();
  wait_for_previous();
  if (row < p.count[r]) {
    const int64_t at = (int64_t)r * p.rows_pad + row;
    const int n = p.n_parts;
    const float2* part = p.part + at * n;
    const float picked = p.z_target[at];
    const int token = p.token_of[at];
    Lse l{-INFINITY, 0.0f};
#pragma unroll 4
    for (int i = lane; i < n; i += 32) l.add(part[i]);
    l.add_warp();
    if (lane == 0) {
      const Target t(l, picked);
      p.norm[at] = norm_of(l, picked, t.grad);
      write_row(p, r, row, t.loss, token);
    }
  }
  finish_block(p, r, gridDim.x);
}

// One block a row: sum and loss as above, then the row's numerators become G in place, bf16.  The target's own value is not P - 1
// but what the sum of the others gives.
// Rows behind the counted ones, up to the next 64, become zeros, since dW's sums run over them.
template <int CTAS>
__global__ void __launch_bounds__(256) scale_kernel(const __grid_constant__ LossParams p) {
  constexpr int kCols = 64 * CTAS;
  extern __shared__ float s_factor[];              // per half tile: 2^64 exp(m) / the row's sum
  __shared__ Lse s_lse[8];
  let_next_start();
  wait_for_previous();
  const int g = blockIdx.y, r = p.r0 + g, row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int count = p.count[r], n = p.n_parts;
  uint4* values = reinterpret_cast<uint4*>(p.g + ((int64_t)g * p.rows_pad + row) * p.v_pitch);
  const int vectors = p.n_tiles * 2 * kCols / 8;
  if (row < count) {
    const int64_t at = (int64_t)r * p.rows_pad + row;
    const float2* part = p.part + at * n;
    const float picked = p.z_target[at];
    const int token = p.token_of[at], target = p.target[at];
    Lse l{-INFINITY, 0.0f};
    for (int i = threadIdx.x; i < n; i += 256) {
      const float2 o = part[i];
      s_factor[i] = o.x;
      l.add(o);
    }
    l.add_warp();
    if (lane == 0) s_lse[warp] = l;
    __syncthreads();
    l = s_lse[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) l.add(make_float2(s_lse[w].top, s_lse[w].sum));
    const Target own(l, picked);
    const RowNorm norm = norm_of(l, picked, own.grad);
    for (int i = threadIdx.x; i < n; i += 256) s_factor[i] = exp_from(s_factor[i], norm.top, kNumeratorBits) * norm.inverse;
    if (threadIdx.x == 0) write_row(p, r, row, own.loss, token);
    __syncthreads();
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += 256) {
      const uint4 u = values[i];
      const float f = s_factor[i * 8 / kCols];
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      float x[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 y = numerators_of(w[k]);
        x[2 * k] = y.x * f;
        x[2 * k + 1] = y.y * f;
      }
      if (i == target / 8) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k == target % 8) x[k] = norm.target;
      }
      values[i] = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    }
  } else if (row < (count + kBlockK - 1) / kBlockK * kBlockK) {
    for (int i = threadIdx.x; i < vectors; i += 256) values[i] = make_uint4(0, 0, 0, 0);
  }
  finish_block(p, r, gridDim.x);
}

// ------------------------------------------------------------------------------------------------ few tokens
// The losses of one or two tokens a replica: the table is read once, so that is what bounds it, and a product of 128 rows
// would leave the tensor cores 126 of them empty.  A warp takes a run of the table's rows, three at a time, a lane 8 elements of
// each per step; hidden states come from L1.  Sums are fp32.  Its arithmetic grows with the tokens, the product's does not.  One replica,
// 50257 rows, replayed from graphs over three tables in turn, with this kernel, and through packing and the product:
//   1 token   width 768: 19.9 and 34 us    width 2048: 41.9 and 59 us    eight replicas of width 768: 105 and 118 us
//   2 tokens             24.0 and 34                   46.5 and 59                                    132 and 118
// and with a form for four tokens, 40.3 and 34 us at three and four, 72 with one for eight.  So two tokens of larger tables than kFewElements,
// in all, take the product.  Two rows at a time: 19.2 us for one token, 27.9 for two; four rows: 21.0 and 24.5.
// 80 registers, which leaves three blocks a SM; up to 28 bytes a thread are spilled for it.
constexpr int kFew = 2, kFewRows = 3;
constexpr int64_t kFewElements = 150000000;

template <int NT>
__global__ void __launch_bounds__(256, 3) few_kernel(const __grid_constant__ LossParams p, const __grid_constant__ PackParams k,
                                                  const __nv_bfloat16* __restrict__ table, int64_t table_stride, int64_t table_row) {
  __shared__ Lse s_lse[8][NT];
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
          target[i] = y;
          hidden[i] = k.hidden + r * k.hidden_stride + t * k.hidden_row;
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && t < k.n_tokens) {
      if (y >= 0) {
        k.target[(int64_t)r * p.rows_pad + count] = y;
        k.token_of[(int64_t)r * p.rows_pad + count] = t;
      } else if (p.token_loss) {
        p.token_loss[r * p.token_loss_stride + t] = 0.0f;
      }
    }
    count += y >= 0;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    k.count[r] = count;
  }
  if (count == 0) return;
  const int64_t w = (int64_t)blockIdx.x * 8 + warp, warps = (int64_t)gridDim.x * 8;
  const int from = (int)(p.vocab * w / warps), to = (int)(p.vocab * (w + 1) / warps);
  const __nv_bfloat16* base = table + r * table_stride;
  Lse l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) l[t] = Lse{-INFINITY, 0.0f};
  for (int v = from; v < to; v += kFewRows) {
    float z[kFewRows][NT];
    const __nv_bfloat16* row[kFewRows];
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      row[i] = base + min(v + i, to - 1) * table_row;   // behind the run's end: its last row again, not counted
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
        if (v + i != target[t]) l[t].add_logit(z[i][t]);
        else if (lane == 0) p.z_target[(int64_t)r * p.rows_pad + t] = z[i][t];
      }
  }
  if (lane == 0)
#pragma unroll
    for (int t = 0; t < NT; ++t) s_lse[warp][t] = l[t];
  __syncthreads();
  if (threadIdx.x < count) {
    Lse all = s_lse[0][threadIdx.x];
    for (int i = 1; i < 8; ++i) all.add(make_float2(s_lse[i][threadIdx.x].top, s_lse[i][threadIdx.x].sum));
    p.part[((int64_t)r * p.rows_pad + threadIdx.x) * p.n_parts + blockIdx.x] = make_float2(all.top, all.sum);
  }
}

// What follows few_kernel: a warp a token, all of its loads under way at once, then the mean.
__global__ void __launch_bounds__(32 * kFew) few_join_kernel(const __grid_constant__ LossParams p) {
  __shared__ float s_loss[kFew];
  let_next_start();
  wait_for_previous();
  const int r = blockIdx.x, t = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int count = p.count[r];
  const int64_t at = (int64_t)r * p.rows_pad + t;
  const float picked = p.z_target[at];             // nothing of these is used behind the counted tokens
  const int token = p.token_of[at];
  Lse l{-INFINITY, 0.0f};
  for (int i0 = 0; i0 < p.n_parts; i0 += 32 * 16) {
    float2 part[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int i = i0 + 32 * k + lane;
      part[k] = t < p.n_tokens && i < p.n_parts ? p.part[at * p.n_parts + i] : make_float2(-INFINITY, 0.0f);
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) l.add(part[k]);
  }
  l.add_warp();
  const float loss = Target(l, picked).loss;
  if (lane == 0) {
    s_loss[t] = loss;
    if (t < count && p.token_loss) p.token_loss[r * p.token_loss_stride + token] = loss;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  double sum = 0.0;
  for (int i = 0; i < count; ++i) sum += (double)s_loss[i];
  const double mean = count > 0 ? sum / (double)count : 0.0;
  if (p.loss_f64) static_cast<double*>(p.loss)[r] = mean; else static_cast<float*>(p.loss)[r] = (float)mean;
}

// dH: adds the partial sums over the vocabulary in their order, scales, rounds once and puts rows back at their tokens.
__global__ void __launch_bounds__(256) join_hidden_kernel(const __grid_constant__ LossParams p) {
  let_next_start();
  wait_for_previous();
  const int g = blockIdx.y, r = p.r0 + g, row = blockIdx.x;
  const int count = p.count[r];
  if (row >= count) return;
  const float scale = (float)(p.grad_scale / (double)(p.of_mean ? count : 1));
  const Out o = p.d_hidden;
  const int64_t to = r * o.stride + (int64_t)p.token_of[(int64_t)r * p.rows_pad + row] * o.row;
  for (int c = threadIdx.x; c < p.width; c += 256) {
    float sum = 0.0f;
    for (int s = 0; s < p.h_splits; ++s) sum += p.slabs[(((int64_t)s * p.n_r + g) * p.rows_pad + row) * p.width + c];
    sum *= scale;
    if (o.f32) static_cast<float*>(o.p)[to + c] = sum;
    else static_cast<__nv_bfloat16*>(o.p)[to + c] = __float2bfloat16_rn(sum);
  }
}

// After G from given gradients: the likely classes' entries.  32 rows a block, a lane each, whose sums the block's warps share.
__global__ void __launch_bounds__(1024) likely_kernel(const __grid_constant__ LossParams p) {
  __shared__ float s_sum[32][33];
  let_next_start();
  wait_for_previous();
  const int r = p.r0 + blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * 32 + lane, certain = p.certain[r];
  if (blockIdx.x * 32 >= certain) return;
  // below 0: in an earlier piece, or not found
  const int v = row < certain ? p.likely[(int64_t)r * p.rows_pad + row] - p.v0 : -1;
  const bool here = v >= 0 && v < p.v_len;
  const int64_t in_group = (int64_t)blockIdx.y * p.rows_pad + row, all = (int64_t)p.g_group * p.rows_pad;
  float sum = 0.0f;
  if (here) {
#pragma unroll 8
    for (int i = warp; i < p.n_parts; i += 32) sum += p.others[i * all + in_group];
  }
  s_sum[warp][lane] = sum;
  __syncthreads();
  sum = s_sum[lane][warp];                         // a warp a row
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __syncthreads();
  if (lane == 0) s_sum[0][warp] = sum;
  __syncthreads();
  if (warp != 0 || !here) return;
  float left = -s_sum[0][lane];
  for (int term = 0; term < p.g_terms; ++term) {
    const __nv_bfloat16 g = __float2bfloat16_rn(left);
    p.g[(term * all + in_group) * p.v_pitch + v] = g;
    left -= __bfloat162float(g);
  }
}

// After the gradients for given ones, which have no losses that could tell: if a wait ran out, the gradients' first elements do.
__global__ void __launch_bounds__(32) poison_grads_kernel(const __grid_constant__ LossParams p) {
  wait_for_previous();
  if (!p.control->status || threadIdx.x >= p.n_replicas) return;
  const auto poison = [&](const Out& o) {
    if (!o.p) return;
    if (o.f32) static_cast<float*>(o.p)[threadIdx.x * o.stride] = NAN;
    else static_cast<__nv_bfloat16*>(o.p)[threadIdx.x * o.stride] = __float2bfloat16_rn(NAN);
  };
  if (p.n_tokens > 0) poison(p.d_hidden);
  poison(p.d_weight);
}

// ------------------------------------------------------------------------------------------------ host side
int check(const char* who, const hdet_token_loss_args* d) {
  if (!d) return fail(HDET_ERR_INVALID_ARG, who, "the descriptor is NULL");
  if (d->n_replicas < 1 || d->n_replicas > HDET_MAX_REPLICAS)
    return fail(HDET_ERR_INVALID_ARG, who, "n_replicas must be in 1..32");
  if (d->n_tokens < 0 || d->n_tokens > HDET_MAX_TOKENS || d->vocab < 1 || d->vocab > HDET_MAX_VOCAB || d->width < 1 ||
      d->width > HDET_MAX_WIDTH)
    return fail(HDET_ERR_INVALID_ARG, who, "n_tokens, vocab or width out of range");
  if (d->target_dtype != HDET_DTYPE_I32 && d->target_dtype != HDET_DTYPE_I64)
    return fail(HDET_ERR_INVALID_ARG, who, "target_dtype must be HDET_DTYPE_I32 or HDET_DTYPE_I64");
  if (d->loss_dtype != HDET_DTYPE_F32 && d->loss_dtype != HDET_DTYPE_F64)
    return fail(HDET_ERR_INVALID_ARG, who, "loss_dtype must be HDET_DTYPE_F32 or HDET_DTYPE_F64");
  if (d->hidden_dtype != HDET_DTYPE_BF16 || d->weight_dtype != HDET_DTYPE_BF16) {
    if (!is_float(d->hidden_dtype) || !is_float(d->weight_dtype))
      return fail(HDET_ERR_INVALID_ARG, who, "hidden_dtype and weight_dtype must be HDET_DTYPE_*");
    return fail(HDET_ERR_UNSUPPORTED, who, "hidden states and table must be HDET_DTYPE_BF16 (hdet_tensor.param_bf16, or a bf16 copy)");
  }
  if ((d->d_hidden && !is_float(d->d_hidden_dtype)) || (d->d_weight && !is_float(d->d_weight_dtype)))
    return fail(HDET_ERR_INVALID_ARG, who, "the gradients' dtypes must be HDET_DTYPE_F32 or HDET_DTYPE_BF16");
  if (d->device < 0) return fail(HDET_ERR_INVALID_ARG, who, "device must be >= 0");
  if (!std::isfinite((float)d->grad_scale)) return fail(HDET_ERR_INVALID_ARG, who, "grad_scale must be finite in fp32");
  if (d->piece_bytes < 0) return fail(HDET_ERR_INVALID_ARG, who, "piece_bytes must be >= 0");
  if (d->hidden_row < d->width || d->weight_row < d->width || (d->d_hidden && d->d_hidden_row < d->width) ||
      (d->d_weight && d->d_weight_row < d->width))
    return fail(HDET_ERR_INVALID_ARG, who, "a row stride is smaller than width");
  const int64_t strides[] = {d->hidden_stride, d->weight_stride, d->target_stride, d->token_loss_stride, d->d_hidden_stride,
                             d->d_weight_stride};
  for (const int64_t s : strides) {
    if (d->n_replicas == 1) break;
    if (s < 0) return fail(HDET_ERR_INVALID_ARG, who, "negative stride");
    if (s > HDET_MAX_REPLICA_STRIDE) return fail(HDET_ERR_INVALID_ARG, who, "a replica stride is out of range");
  }
  if (std::max({d->hidden_row, d->weight_row, d->d_hidden ? d->d_hidden_row : 0, d->d_weight ? d->d_weight_row : 0}) > HDET_MAX_ROW_STRIDE)
    return fail(HDET_ERR_INVALID_ARG, who, "a row stride is out of range");
  return HDET_OK;
}

int check_pointers(const char* who, const hdet_token_loss_args* d) {
  if (!d->weight || !d->loss || (d->n_tokens > 0 && (!d->hidden || !d->targets)))
    return fail(HDET_ERR_INVALID_ARG, who, "a pointer is NULL");
  const auto span = [&](int64_t rows, int64_t row) { return rows > 0 ? (rows - 1) * row + d->width : 0; };
  if (d->n_replicas > 1) {
    if ((d->hidden_stride && d->hidden_stride < span(d->n_tokens, d->hidden_row)) ||
        (d->weight_stride && d->weight_stride < span(d->vocab, d->weight_row)) ||
        (d->target_stride && d->target_stride < d->n_tokens) ||
        (d->token_loss && d->token_loss_stride < d->n_tokens) ||
        (d->d_hidden && d->d_hidden_stride < span(d->n_tokens, d->d_hidden_row)) ||
        (d->d_weight && d->d_weight_stride < span(d->vocab, d->d_weight_row)))
      return fail(HDET_ERR_INVALID_ARG, who, "a replica stride is smaller than one replica");
  }
  // In the hidden states' own buffer every row of d_hidden has to lie on its own hidden state's: other rows are still to be read.
  if (d->d_hidden && d->d_hidden == d->hidden && d->n_tokens > 0 &&
      (d->d_hidden_dtype != HDET_DTYPE_BF16 || d->d_hidden_row != d->hidden_row || (d->n_replicas > 1 && d->d_hidden_stride != d->hidden_stride)))
    return fail(HDET_ERR_INVALID_ARG, who, "d_hidden in the place of the hidden states needs their dtype and strides");
  if (!aligned(d->hidden, 2) || !aligned(d->weight, 2) || !aligned(d->targets, d->target_dtype == HDET_DTYPE_I64 ? 8 : 4) ||
      !aligned(d->loss, d->loss_dtype == HDET_DTYPE_F64 ? 8 : 4) || !aligned(d->token_loss, 4) ||
      (d->d_hidden && !aligned(d->d_hidden, elem_size(d->d_hidden_dtype))) ||
      (d->d_weight && !aligned(d->d_weight, elem_size(d->d_weight_dtype))))
    return fail(HDET_ERR_ALIGN, who, "a pointer is not aligned to its element type");
  return HDET_OK;
}

// Whether the table's boxes can be copied from where it is.
bool table_fits(const hdet_token_loss_args* d) {
  const bool many = d->n_replicas > 1;
  return aligned(d->weight, 16) && d->weight_row % 8 == 0 && (!many || d->weight_stride % 8 == 0);
}

// Larger pieces mean fewer passes over the hidden states and, where a replica's G no longer fits, no second forming of the logits.  In ms, for
// pieces of 64, 128, 256, 512 and 1024 MB: 16 x 1024 tokens x 768 5.46, 4.66, 4.46, 4.33, 4.22; 8 x 2048 x 2048 11.4, 11.1, 8.83, 8.82, 8.73;
// fp32 gradients of 4 x 1024 x 768 3.21, 2.88, 2.73, 2.68, 2.66.  Twice the memory beyond 512 MB gives 1 - 3 %.
constexpr int64_t kDefaultPieceBytes = 512ll << 20;
constexpr int kTermsF32 = 3;     // bf16 numbers that hold G for fp32 gradients
constexpr int64_t kMaxScaleTiles = 4096;      // scale_kernel keeps two factors a tile in shared memory (32 KB)
constexpr int64_t kFewBlocks = 148 * 3;         // blocks of few_kernel that are resident at once
constexpr int kSlots = 74;       // pairs of SMs of a B200: tiles that run at once (another count would change times only)

// Sizes, launches and the workspace's layout; host arithmetic only, the same for the size query and the call.
struct Plan {
  int ctas, tile;
  int64_t rows_pad, packed_row, m_tiles, n_tiles;
  bool grads;
  int h_terms, w_terms, g_terms;  // terms of G in each product, and in the workspace
  bool numerators;                // the logits are formed once: their exponentials wait in the workspace for lse
  bool few;                       // few_kernel takes the place of packing and product
  int64_t n_parts;                // parts of a row's sum of exp
  int64_t group;                  // replicas per launch
  int64_t piece;                  // rows of the table per launch (a multiple of the tile)
  int64_t n_pieces, h_len, h_splits;
  bool h_slabs;
  bool pack_table;
  int64_t off_count, off_target, off_token, off_z, off_norm, off_part, off_loss, off_certain, off_likely, off_others, off_hidden, off_table, off_g,
      off_slabs, total;
};

// `given`: G comes from given gradients; there are no losses and nothing waits for a normaliser.
Plan plan_of(const hdet_token_loss_args* d, bool given) {
  Plan q{};
  const int64_t R = d->n_replicas, T = d->n_tokens, V = d->vocab, D = d->width;
  // Pairs share operands, single CTAs make four times as many tiles.  1 x 1024 tokens x 50257 (width 768), loss and bf16
  // gradients: 293 us in pairs, 348 in singles; 1 x 256 x 4099 (512): 42 and 39; 1 x 150 x 50257 (768): 125 and 110.
  q.ctas = T <= 192 || R * div_up(T, 256) * div_up(V, 256) < 64 ? 1 : 2;
  q.tile = 128 * q.ctas;
  q.rows_pad = round_up(T > 0 ? T : 1, q.tile);
  q.packed_row = round_up(D, 8);
  q.m_tiles = q.rows_pad / q.tile;
  q.n_tiles = div_up(V, q.tile);
  q.grads = d->d_hidden || d->d_weight;
  q.h_terms = d->d_hidden && d->d_hidden_dtype == HDET_DTYPE_F32 ? kTermsF32 : 1;
  q.w_terms = d->d_weight && d->d_weight_dtype == HDET_DTYPE_F32 ? kTermsF32 : 1;
  q.g_terms = q.h_terms > q.w_terms ? q.h_terms : q.w_terms;
  q.pack_table = !table_fits(d);
  q.few = !q.grads && T <= kFew && T > 0 && (T == 1 || R * V * D <= kFewElements) && !q.pack_table && D % 8 == 0 && aligned(d->hidden, 16) && d->hidden_row % 8 == 0 &&
          (R == 1 || d->hidden_stride % 8 == 0);
  const int64_t most = div_up(V, 8 * kFewRows), blocks = kFewBlocks / R;
  const int64_t few_parts = blocks < 1 ? 1 : blocks < most ? blocks : most;
  q.n_parts = q.few ? few_parts : 2 * q.n_tiles;
  if (q.grads) {
    const int64_t budget = d->piece_bytes ? d->piece_bytes : kDefaultPieceBytes;
    const int64_t v_all = q.n_tiles * q.tile, per_row = q.rows_pad * 2 * q.g_terms;
    const int64_t fit = budget / (per_row * v_all);
    if (fit >= 1) {
      const int64_t groups = div_up(R, fit);
      q.group = div_up(R, groups);
      q.piece = v_all;
    } else {
      q.group = 1;
      int64_t tiles = budget / (per_row * q.tile);
      if (tiles < 1) tiles = 1;
      tiles = div_up(q.n_tiles, div_up(q.n_tiles, tiles));       // equal pieces
      q.piece = tiles * q.tile;
    }
    q.n_pieces = div_up(v_all, q.piece);
    // With all of a replica's G in the workspace, and G in bf16, its place can hold the numerators until lse is known: a pass
    // over 2 bytes a logit in place of 2 x width operations.  (16 x 1024 tokens of width 768: 4.16 ms, with the logits formed
    // twice 4.67; 8 x 2048 of width 2048: 8.39 and 10.1.)
    q.numerators = !given && q.n_pieces == 1 && q.g_terms == 1 && q.n_tiles <= kMaxScaleTiles;
    if (d->d_hidden) {
      // dH's sums run over the piece, dW's over the tokens: dH has few tiles and long sums.  Cut into parts, it ends with the
      // rest of the launch's work; every part more costs a pass over fp32 partial sums, about two steps a tile.  The cut taken
      // is the one with the shortest end: rounds of dH's jobs, or an equal share of all the work where that is longer.
      const int64_t all = div_up(q.piece, kBlockK), h_tiles = q.group * q.m_tiles * div_up(D, q.tile);
      const int64_t w_tiles = d->d_weight ? q.group * (q.piece / q.tile) * div_up(D, q.tile) : 0;
      const int64_t work = h_tiles * all * q.h_terms + w_tiles * div_up(T, kBlockK) * q.w_terms;
      const int64_t slots = kSlots * (3 - q.ctas);
      const double share = (double)work / (double)slots;
      double best = 0.0;
      for (int64_t parts = 1; parts <= 64; ++parts) {
        if (best != 0.0 && share >= 0.98 * best) break;        // no cut ends before the equal share
        const int64_t len = div_up(all, parts), n = div_up(all, len);
        if (n != parts || (parts > 1 && len < 8)) continue;
        const double rounds = (double)(div_up(h_tiles * n, slots) * len * q.h_terms);
        const double end = (rounds > share ? rounds : share) + (n > 1 ? 2.0 * (double)(h_tiles * n) / (double)slots : 0.0);
        if (best == 0.0 || end < 0.98 * best) {
          best = end;
          q.h_len = len;
          q.h_splits = n;
        }
      }
      q.h_slabs = q.h_splits > 1 || q.n_pieces > 1;
    }
  }
  int64_t at = round_up(sizeof(Control), 256);
  const auto take = [&](int64_t bytes) { const int64_t o = at; at = round_up(at + bytes, 256); return o; };
  q.off_count = take(4 * R);
  q.off_target = take(4 * R * q.rows_pad);
  q.off_token = take(4 * R * q.rows_pad);
  q.off_norm = take(sizeof(RowNorm) * R * q.rows_pad);
  if (!given) {
    q.off_z = take(4 * R * q.rows_pad);
    // room for either kernel's parts: which one runs depends on the hidden states' address, and the size does not
    q.off_part = take(8 * R * std::max(2 * q.n_tiles, !q.grads && T <= kFew ? few_parts : 0) * q.rows_pad);
    q.off_loss = take(4 * R * q.rows_pad);
  } else if (q.grads) {
    q.off_certain = take(4 * R);
    q.off_likely = take(4 * R * q.rows_pad);
    q.off_others = take(4 * q.group * q.rows_pad * 2 * q.n_tiles);
  }
  q.off_hidden = take(2 * R * q.rows_pad * q.packed_row);
  if (q.pack_table) q.off_table = take(2 * (d->n_replicas > 1 && d->weight_stride ? R : 1) * V * q.packed_row);
  if (q.grads) {
    q.off_g = take(2 * q.g_terms * q.group * q.rows_pad * q.piece);
    if (q.h_slabs) q.off_slabs = take(4 * q.h_splits * q.group * q.rows_pad * D);
  }
  q.total = at;
  return q;
}

// The most that a call with up to n_tokens tokens needs.  A shorter batch can need more than a longer one: more of its replicas share a
// launch, or its sums are cut into more parts.  The plan is the same for tokens up to the same multiple of 64 (but for the few that
// have a kernel of their own).
int64_t workspace_of(const hdet_token_loss_args* d, bool given) {
  hdet_token_loss_args a = *d;
  int64_t most = plan_of(d, given).total;
  for (a.n_tokens = kFew; a.n_tokens < d->n_tokens; a.n_tokens = a.n_tokens == kFew ? 64 : a.n_tokens + 64)
    most = std::max(most, plan_of(&a, given).total);
  return most;
}

// Once per device: the kernels' shared-memory sizes and its SM count.
cudaError_t prepare(int device, int* sms) {
  const void* kernels[] = {
#define HDET_PHASES(ctas, sums)                                                                              \
  (const void*)gemm_kernel<ctas, kStats, sums>, (const void*)gemm_kernel<ctas, kNumerators, sums>,           \
      (const void*)gemm_kernel<ctas, kProbs, sums>, (const void*)gemm_kernel<ctas, kGrads, sums>,         \
      (const void*)gemm_kernel<ctas, kGiven, sums>
      HDET_PHASES(1, false), HDET_PHASES(1, true), HDET_PHASES(2, false), HDET_PHASES(2, true)};
#undef HDET_PHASES
  return prepare_device(device, sms, kernels, kGemmSmem);
}

// Steps of 64 summed by the tensor cores at a time.  fp32 gradients, and the logits for them: 8 (errors of 4e-8 to 9e-7 of a gradient's
// norm; 4 steps 3e-8 to 5e-7, 14 % slower; 16 steps up to 1.9e-6, 6 % faster).  Other logits: 16.  A likely target's products
// mostly have one sign, so their cuts add up: at a width of 2048 and a target's logit of 24 the loss of a token is 3.4e-5 of its value off
// with 64 steps, 1.6e-5 with 16, 0.8e-5 with 8 (as an fp32 product); 8 x 2048 tokens with bf16 gradients take 8.35, 8.41 and 8.80 ms, 4 x 1024
// of width 768 with fp32 gradients 2.56, 2.54 and 2.63.  bf16 gradients: 256, 3e-5, far below their rounding.
constexpr int kChunkLogits = 16, kChunkF32 = 8, kChunkBf16 = 256;
constexpr int kWholeBf16 = 1024;   // bf16 gradients up to this many steps are not cut at all: 1e-4

template <int PHASE>
cudaError_t launch_gemm(LossParams& p, int ctas, int64_t tiles, int sms, cudaStream_t st) {
  if (tiles == 0) return cudaSuccess;
  const int64_t clusters = tiles < sms / ctas ? tiles : sms / ctas;
  p.jobs = (int)tiles;
  // the longest sum of this launch, and what it is cut into
  const int64_t longest = PHASE != kGrads ? div_up(p.width, kBlockK)
                                          : std::max<int64_t>(p.h_jobs ? (int64_t)p.h_len * p.h_terms : 0,
                                                              p.w_tiles_m ? div_up(p.n_tokens, kBlockK) * p.w_terms : 0);
  p.chunk = p.g_terms > 1 ? kChunkF32 : PHASE != kGrads ? kChunkLogits : kChunkBf16;
  const bool sums = longest > (PHASE == kGrads && p.g_terms == 1 ? kWholeBf16 : p.chunk);
  const dim3 grid((unsigned)(clusters * ctas));
  const auto kernel = ctas == 1 ? (sums ? gemm_kernel<1, PHASE, true> : gemm_kernel<1, PHASE, false>)
                                : (sums ? gemm_kernel<2, PHASE, true> : gemm_kernel<2, PHASE, false>);
  const cudaError_t e = launch(kernel, grid, kGemmThreads, kGemmSmem, ctas, st, p);
  p.first_ticket += (unsigned)tiles;
  return e;
}

Out out_of(void* p, int dtype, int64_t stride, int64_t row, int64_t width, bool many, bool accumulate) {
  Out o{};
  o.p = p;
  o.f32 = dtype == HDET_DTYPE_F32;
  o.stride = many ? stride : 0;
  o.row = row;
  o.accumulate = accumulate;
  const int per16 = 16 / elem_size(dtype);
  o.vec = aligned(p, 16) && row % per16 == 0 && o.stride % per16 == 0 && width % per16 == 0;
  return o;
}

}  // namespace
}  // namespace hdet

using namespace hdet;

extern "C" HDET_API int hdet_token_loss_workspace(const hdet_token_loss_args* d, int64_t* bytes) {
  const char* who = "hdet_token_loss_workspace";
  if (!bytes) return fail(HDET_ERR_INVALID_ARG, who, "bytes is NULL");
  *bytes = 0;
  if (const int rc = check(who, d)) return rc;
  *bytes = workspace_of(d, false);
  return HDET_OK;
}

namespace hdet {
namespace {

// Behind the checks of the descriptor.  `given`: no loss, and the gradients for given ones of log probabilities and entropies.
int token_loss(const char* who, const hdet_token_loss_args* d, const ScoreGiven* given, void* workspace, int64_t workspace_bytes, void* stream,
               bool selftest) {
  const Plan q = plan_of(d, given != nullptr);
  if (!workspace || workspace_bytes < q.total)
    return fail(HDET_ERR_INVALID_ARG, who, given ? "the workspace is NULL or smaller than hdet_token_scores_grad_workspace says"
                                                 : "the workspace is NULL or smaller than hdet_token_loss_workspace says");
  if (!aligned(workspace, 256)) return fail(HDET_ERR_ALIGN, who, "the workspace is not 256-byte aligned");
  if (q.m_tiles * q.n_tiles * d->n_replicas * q.ctas > INT32_MAX || q.rows_pad * q.packed_row * 2 >= (1ll << 40) ||
      d->weight_row * d->vocab * 2 >= (1ll << 40) || (d->n_replicas > 1 && d->weight_stride * 2 >= (1ll << 40)))
    return fail(HDET_ERR_UNSUPPORTED, who, "too many tiles, or a stride of 2^40 bytes or more");
  DeviceScope scope(d->device);
  if (scope.err != cudaSuccess) return fail_cuda(who, scope.err);
  int sms = 0;
  cudaError_t e = prepare(d->device, &sms);
  if (e != cudaSuccess) return fail_cuda(who, e);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const bool many = d->n_replicas > 1;
  const bool shared_table = !many || d->weight_stride == 0;

  LossParams p{};
  p.n_replicas = d->n_replicas;
  p.vocab = (int)d->vocab; p.width = (int)d->width; p.n_tokens = (int)d->n_tokens; p.rows_pad = (int)q.rows_pad;
  p.weight_shared = shared_table;
  p.grad_scale = d->grad_scale;
  p.of_mean = !given;
  p.wait_limit = selftest ? kSelftestLimitCycles : bulk::kWaitLimitCycles;
  p.withhold = selftest;
  p.count = reinterpret_cast<int*>(ws + q.off_count);
  p.target = reinterpret_cast<int*>(ws + q.off_target);
  p.token_of = reinterpret_cast<int*>(ws + q.off_token);
  p.norm = reinterpret_cast<RowNorm*>(ws + q.off_norm);
  if (!given) {
    p.z_target = reinterpret_cast<float*>(ws + q.off_z);
    p.part = reinterpret_cast<float2*>(ws + q.off_part);
    p.row_loss = reinterpret_cast<float*>(ws + q.off_loss);
  } else if (given->d_entropy.p) {
    p.certain = reinterpret_cast<int*>(ws + q.off_certain);
    p.likely = reinterpret_cast<int*>(ws + q.off_likely);
    p.others = reinterpret_cast<float*>(ws + q.off_others);
  }
  p.token_loss = static_cast<float*>(d->token_loss);
  p.token_loss_stride = many ? d->token_loss_stride : 0;
  p.loss = d->loss;
  p.loss_f64 = d->loss_dtype == HDET_DTYPE_F64;
  p.control = reinterpret_cast<Control*>(ws);
  if (d->d_hidden) p.d_hidden = out_of(d->d_hidden, d->d_hidden_dtype, d->d_hidden_stride, d->d_hidden_row, d->width, many, false);
  if (d->d_weight) p.d_weight = out_of(d->d_weight, d->d_weight_dtype, d->d_weight_stride, d->d_weight_row, d->width, many, d->accumulate != 0);

  // packing
  PackParams k{};
  k.hidden = static_cast<const __nv_bfloat16*>(d->hidden);
  k.hidden_stride = many ? d->hidden_stride : 0;
  k.hidden_row = d->hidden_row;
  k.targets = d->targets;
  k.target_stride = many ? d->target_stride : 0;
  k.wide = d->target_dtype == HDET_DTYPE_I64;
  k.hidden_vec = aligned(d->hidden, 16) && d->hidden_row % 8 == 0 && k.hidden_stride % 8 == 0 && d->width % 8 == 0;
  k.d_hidden = p.d_hidden;
  k.d_hidden_vec = p.d_hidden.vec;
  k.n_tokens = p.n_tokens; k.vocab = p.vocab; k.width = p.width; k.rows_pad = p.rows_pad; k.row_tile = q.tile;
  k.packed_row = (int)q.packed_row;
  k.packed = reinterpret_cast<__nv_bfloat16*>(ws + q.off_hidden);
  k.count = const_cast<int*>(p.count);
  k.target = const_cast<int*>(p.target);
  k.token_of = const_cast<int*>(p.token_of);
  k.token_loss = p.token_loss;
  k.token_loss_stride = p.token_loss_stride;
  k.control = p.control;
  const __nv_bfloat16* table = static_cast<const __nv_bfloat16*>(d->weight);
  int64_t table_row = d->weight_row, table_stride = shared_table ? d->weight_row * d->vocab : d->weight_stride;
  const int tables = shared_table ? 1 : d->n_replicas;
  p.n_parts = (int)q.n_parts;
  if (q.few) {
    if (selftest) return fail(HDET_ERR_UNSUPPORTED, who, "the kernel for so few tokens waits for nothing");
    const dim3 grid((unsigned)q.n_parts, d->n_replicas);
    const int64_t stride = shared_table ? 0 : table_stride;
    e = launch(d->n_tokens == 1 ? few_kernel<1> : few_kernel<2>, grid, 256, 0, 1, st, p, k, table,
               stride, table_row);
    if (e == cudaSuccess) e = launch(few_join_kernel, dim3(d->n_replicas), 32 * kFew, 0, 1, st, p);
    return e == cudaSuccess ? HDET_OK : fail_cuda(who, e);
  }
  const int64_t pack_rows = round_up(div_up(d->n_tokens > 0 ? d->n_tokens : 1, kPackBlocks), 8);
  const unsigned pack_blocks = (unsigned)(d->n_tokens > 0 ? div_up(d->n_tokens, pack_rows) : 1);
  const dim3 pack_grid(pack_blocks, d->n_replicas);
  if (given) {
    ScoreGiven g = *given;
    g.norm = const_cast<RowNorm*>(p.norm);
    g.certain = const_cast<int*>(p.certain);
    g.likely = p.likely;
    e = launch(pack_kernel<kPackGiven, ScoreGiven>, pack_grid, 256, 0, 1, st, k, (int)pack_rows, g);
  } else {
    e = launch(pack_kernel<kPackLoss, int>, pack_grid, 256, 0, 1, st, k, (int)pack_rows, 0);
  }
  if (e != cudaSuccess) return fail_cuda(who, e);

  if (q.pack_table) {
    __nv_bfloat16* packed = reinterpret_cast<__nv_bfloat16*>(ws + q.off_table);
    e = launch_pack_table(table, shared_table ? 0 : d->weight_stride, table_row, p.vocab, p.width, k.packed_row, tables, packed, st);
    if (e != cudaSuccess) return fail_cuda(who, e);
    table = packed;
    table_row = q.packed_row;
    table_stride = q.packed_row * d->vocab;
  }
  bool maps = encode(&p.hidden, k.packed, d->width, q.rows_pad, d->n_replicas, q.packed_row, q.rows_pad * q.packed_row) &&
              encode(&p.weight, table, d->width, d->vocab, tables, table_row, table_stride);
  if (maps && q.grads) {
    p.g = reinterpret_cast<__nv_bfloat16*>(ws + q.off_g);
    p.g_terms = q.g_terms;
    p.g_group = (int)q.group;
    maps = encode(&p.grad, p.g, q.piece, q.rows_pad, q.g_terms * q.group, q.piece, q.rows_pad * q.piece);
  }
  if (!maps) return fail(HDET_ERR_CUDA, who, "the driver refused a tensor map");

  // the loss
  p.r0 = 0; p.n_r = d->n_replicas;
  p.v0 = 0; p.v_len = p.vocab; p.v_pitch = (int)q.piece;
  p.m_tiles = (int)q.m_tiles; p.n_tiles = (int)q.n_tiles;
  const bool any = d->n_tokens > 0;
  if (!q.numerators && !given) {
    if (any) e = launch_gemm<kStats>(p, q.ctas, q.m_tiles * q.n_tiles * d->n_replicas, sms, st);
    if (e == cudaSuccess) e = launch(join_kernel, dim3((unsigned)(q.rows_pad / 8), d->n_replicas), 256, 0, 1, st, p);
  }
  if (e != cudaSuccess) return fail_cuda(who, e);

  // the gradients, piece by piece
  if (q.grads) {
    p.slabs = reinterpret_cast<float*>(ws + q.off_slabs);
    p.h_terms = q.h_terms; p.w_terms = q.w_terms;
    p.h_slabs = q.h_slabs;
    p.h_splits = (int)q.h_splits; p.h_len = (int)q.h_len;
    p.h_tiles_m = (int)q.m_tiles; p.h_tiles_n = p.w_tiles_n = (int)div_up(d->width, q.tile);
    const auto take_piece = [&](int64_t piece) {
      p.v0 = (int)(piece * q.piece);
      p.v_len = (int)(d->vocab - p.v0 < q.piece ? d->vocab - p.v0 : q.piece);
      p.n_tiles = (int)div_up(p.v_len, q.tile);
    };
    for (int64_t r0 = 0; r0 < d->n_replicas; r0 += q.group) {
      p.r0 = (int)r0;
      p.n_r = (int)(d->n_replicas - r0 < q.group ? d->n_replicas - r0 : q.group);
      // The likely classes' entries need the others of the whole vocabulary: with more than one piece, the certain rows' logits are formed once more
      // (2 x 2048 tokens x 50257 of width 768, fp32 gradients in two pieces, 60 % of the rows certain: 2.15 -> 2.50 ms).
      if (p.certain && any && q.n_pieces > 1) {
        p.sums_only = true;
        p.count = p.certain;
        for (int64_t piece = 0; e == cudaSuccess && piece < q.n_pieces; ++piece) {
          take_piece(piece);
          e = launch_gemm<kGiven>(p, q.ctas, (int64_t)p.n_r * p.m_tiles * p.n_tiles, sms, st);
        }
        p.sums_only = false;
        p.count = k.count;
        if (e != cudaSuccess) return fail_cuda(who, e);
      }
      for (int64_t piece = 0; piece < q.n_pieces; ++piece) {
        take_piece(piece);
        p.w_tiles_m = d->d_weight ? p.n_tiles : 0;
        p.h_jobs = d->d_hidden && any ? p.h_splits * p.n_r * p.h_tiles_m * p.h_tiles_n : 0;
        p.h_add = piece > 0;
        const int64_t tiles = (int64_t)p.n_r * p.m_tiles * p.n_tiles;
        if (given) {
          if (any) e = launch_gemm<kGiven>(p, q.ctas, tiles, sms, st);
          if (e == cudaSuccess && any && p.certain) e = launch(likely_kernel, dim3((unsigned)(q.rows_pad / 32), p.n_r), 1024, 0, 1, st, p);
        } else if (!q.numerators) {
          if (any) e = launch_gemm<kProbs>(p, q.ctas, tiles, sms, st);
        } else {
          if (any) e = launch_gemm<kNumerators>(p, q.ctas, tiles, sms, st);
          if (e == cudaSuccess) {
            const dim3 grid((unsigned)q.rows_pad, p.n_r);
            const size_t factors = sizeof(float) * 2 * p.n_tiles;
            e = launch(q.ctas == 1 ? scale_kernel<1> : scale_kernel<2>, grid, 256, factors, 1, st, p);
          }
        }
        if (e == cudaSuccess)
          e = launch_gemm<kGrads>(p, q.ctas, p.h_jobs + (int64_t)p.n_r * p.w_tiles_m * p.w_tiles_n, sms, st);
        if (e != cudaSuccess) return fail_cuda(who, e);
      }
      if (d->d_hidden && any && q.h_slabs)
        e = launch(join_hidden_kernel, dim3((unsigned)q.rows_pad, p.n_r), 256, 0, 1, st, p);
      if (e != cudaSuccess) return fail_cuda(who, e);
    }
    if (given) e = launch(poison_grads_kernel, dim3(1), 32, 0, 1, st, p);
    if (e != cudaSuccess) return fail_cuda(who, e);
  }
  return HDET_OK;
}

int checked_token_loss(const char* who, const hdet_token_loss_args* d, void* workspace, int64_t workspace_bytes, void* stream, bool selftest) {
  TraceRange trace(who);
  if (const int rc = check(who, d)) return rc;
  if (const int rc = check_pointers(who, d)) return rc;
  return token_loss(who, d, nullptr, workspace, workspace_bytes, stream, selftest);
}

// The part of a call for given gradients that it has in common with the loss's.
hdet_token_loss_args loss_args(const hdet_token_scores_args* d) {
  hdet_token_loss_args a{};
  a.hidden = d->hidden; a.weight = d->weight; a.targets = d->targets;
  a.d_hidden = d->d_hidden; a.d_weight = d->d_weight;
  a.n_tokens = d->n_tokens; a.vocab = d->vocab; a.width = d->width;
  a.hidden_stride = d->hidden_stride; a.hidden_row = d->hidden_row;
  a.weight_stride = d->weight_stride; a.weight_row = d->weight_row;
  a.target_stride = d->target_stride;
  a.d_hidden_stride = d->d_hidden_stride; a.d_hidden_row = d->d_hidden_row;
  a.d_weight_stride = d->d_weight_stride; a.d_weight_row = d->d_weight_row;
  a.grad_scale = 1.0;
  a.piece_bytes = d->piece_bytes;
  a.n_replicas = d->n_replicas;
  a.hidden_dtype = d->hidden_dtype; a.weight_dtype = d->weight_dtype; a.target_dtype = d->target_dtype;
  a.d_hidden_dtype = d->d_hidden_dtype; a.d_weight_dtype = d->d_weight_dtype;
  a.accumulate = d->accumulate;
  a.device = d->device;
  return a;
}

}  // namespace
}  // namespace hdet

extern "C" HDET_API int hdet_token_loss(const hdet_token_loss_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return checked_token_loss("hdet_token_loss", d, workspace, workspace_bytes, stream, false);
}

extern "C" HDET_API int hdet_selftest_token_loss_wait(const hdet_token_loss_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return checked_token_loss("hdet_selftest_token_loss_wait", d, workspace, workspace_bytes, stream, true);
}

extern "C" HDET_API int hdet_token_scores_grad_workspace(const hdet_token_scores_args* d, int64_t* bytes) {
  const char* who = "hdet_token_scores_grad_workspace";
  if (!bytes) return fail(HDET_ERR_INVALID_ARG, who, "bytes is NULL");
  *bytes = 0;
  if (const int rc = check_token_scores(who, d, true)) return rc;
  const hdet_token_loss_args a = loss_args(d);
  *bytes = workspace_of(&a, true);
  return HDET_OK;
}

namespace {

int token_scores_grad(const char* who, const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream, bool selftest) {
  TraceRange trace(who);
  if (const int rc = check_token_scores(who, d, true)) return rc;
  if (const int rc = check_token_scores_pointers(who, d, true)) return rc;
  const bool many = d->n_replicas > 1;
  const auto per_token = [&](const void* p, int64_t stride) { return PerToken<const float>{static_cast<const float*>(p), many ? stride : 0}; };
  const ScoreGiven given{per_token(d->lse, d->lse_stride), per_token(d->targets ? d->logprob : nullptr, d->logprob_stride),
                         per_token(d->entropy, d->entropy_stride), per_token(d->d_logprob, d->d_logprob_stride),
                         per_token(d->d_entropy, d->d_entropy_stride), nullptr, nullptr, nullptr};
  const hdet_token_loss_args a = loss_args(d);
  return token_loss(who, &a, &given, workspace, workspace_bytes, stream, selftest);
}

}  // namespace

extern "C" HDET_API int hdet_token_scores_grad(const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return token_scores_grad("hdet_token_scores_grad", d, workspace, workspace_bytes, stream, false);
}

extern "C" HDET_API int hdet_selftest_token_scores_grad_wait(const hdet_token_scores_args* d, void* workspace, int64_t workspace_bytes, void* stream) {
  return token_scores_grad("hdet_selftest_token_scores_grad_wait", d, workspace, workspace_bytes, stream, true);
}
