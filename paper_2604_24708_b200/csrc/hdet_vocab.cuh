// What the operators on hidden states and a large table share: packing of the counted tokens, the accumulator's columns in a
// reader's registers, tensor maps, and the host's checks.
#pragma once
#include <cuda_bf16.h>

#include <cmath>
#include <cstdio>
#include <mutex>

#include "../../include/hdet.h"
#include "hdet_internal.h"
#include "hdet_launch.cuh"
#include "hdet_umma.cuh"

namespace hdet {
namespace {

using namespace hdet::umma;

constexpr float kLog2e = 1.4426950408889634f;
constexpr long long kDrainCycles = 20000000ll;          // 10 ms: thousands of times what a copy or a product takes

__host__ __device__ constexpr int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ constexpr int64_t round_up(int64_t a, int64_t b) { return div_up(a, b) * b; }

struct Control {            // first bytes of the workspace; zeroed by pack_kernel (but for `splits`)
  unsigned status;          // a bounded wait ran out
  unsigned ticket;          // tiles handed out by all product kernels of the call so far
  unsigned done[HDET_MAX_REPLICAS];   // blocks of join_kernel that have finished
  int splits;               // parts of the vocabulary that score jobs were made of
};

struct Out {                // a gradient
  void* p;
  int64_t stride, row;
  int f32, accumulate, vec; // vec: rows start and end on 16-byte boundaries
};

// What turns a row's logits into G.  For the loss: inverse * exp(z - top), and the target's own value.  For given gradients of log
// probability and entropy: -exp(z - top) (inverse + slope (z - top)), and the target's own.
struct alignas(16) RowNorm {
  float top, inverse, target, slope;
};

// ------------------------------------------------------------------------------------------------ columns
// Boxes per CTA for a tile with `left` columns from its first to the end.
template <int CTAS>
__device__ __forceinline__ int boxes_for(int left) { return left > 64 * CTAS ? 2 : 1; }

template <int CTAS>
struct Columns {            // of one row: half of a tile's columns
  float x[CTAS][2][32];
};
template <>
struct Columns<0> {};

template <int CTAS>
__device__ __forceinline__ void clear(Columns<CTAS>& acc) {
#pragma unroll
  for (int i = 0; i < 64 * CTAS; ++i) acc.x[i / 64][i / 32 % 2][i % 32] = 0.0f;
}

// The accumulator's columns from `tmem` on, in the place of what acc holds, or added to it.
template <int CTAS>
__device__ __forceinline__ void take_columns(uint32_t tmem, Columns<CTAS>& acc, bool add) {
  __syncwarp();
  if (!add) {
#pragma unroll
    for (int i = 0; i < 2 * CTAS; ++i) tmem_load32(tmem + 32 * i, acc.x[i / 2][i % 2]);
#pragma unroll
    for (int i = 0; i < 2 * CTAS; ++i) tmem_load_wait(acc.x[i / 2][i % 2]);
  } else {
#pragma unroll
    for (int i = 0; i < 4 * CTAS; ++i) {
      float x[16];
      tmem_load16(tmem + 16 * i, x);
      tmem_load_wait(x);
#pragma unroll
      for (int k = 0; k < 16; ++k) acc.x[i / 4][i / 2 % 2][16 * (i % 2) + k] += x[k];
    }
  }
}

// Where an epilogue finds its columns: in the accumulator (SUMS false: one chunk, read 64 columns at a time, which leaves the
// kernel's registers to the loads), or in registers.
template <int CTAS, bool SUMS>
struct Source {
  uint32_t tmem;            // the reader's lanes, at the first column of its half
  Columns<CTAS>* acc;
  bool empty;               // nothing was summed
  // Columns c .. c + 63: those in registers themselves, or `x` with what the accumulator holds.
  __device__ __forceinline__ float (&get(int c, float (&x)[2][32]) const)[2][32] {
    if constexpr (SUMS) {
      return acc->x[c / 64];
    } else {
      if (empty) {
#pragma unroll
        for (int i = 0; i < 64; ++i) x[i / 32][i % 32] = 0.0f;
      } else {
        __syncwarp();
        tmem_load32(tmem + c, x[0]);
        tmem_load32(tmem + c + 32, x[1]);
        tmem_load_wait(x[0]);
        tmem_load_wait(x[1]);
      }
      return x;
    }
  }
};

// exp(x - top) 2^shift.  The subtraction comes first: x log2(e) - top log2(e) in one fma, with the second product rounded, is off by up to
// 2^-24 of the logits themselves, all of a row by the same factor: the gradient of a target with P = 0.9998 was 2 % off for it, one with
// P = 0.999999 by several times its value.
__device__ __forceinline__ float exp_from(float x, float top, float shift = 0.0f) { return exp2_fast(fmaf(x - top, kLog2e, shift)); }

__device__ __forceinline__ float largest(const float (&x)[2][32]) {
  float top[4] = {x[0][0], x[0][1], x[1][0], x[1][1]};
#pragma unroll
  for (int i = 2; i < 32; i += 2) {
    top[0] = fmaxf(top[0], x[0][i]); top[1] = fmaxf(top[1], x[0][i + 1]);
    top[2] = fmaxf(top[2], x[1][i]); top[3] = fmaxf(top[3], x[1][i + 1]);
  }
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

// Columns at or behind the vocabulary's end become -inf (nothing of theirs is left in exp).
__device__ __forceinline__ void cut_columns(float (&x)[2][32], int v, int vocab) {
  if (v + 64 <= vocab) return;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (v + i >= vocab) x[0][i] = -INFINITY;
    if (v + 32 + i >= vocab) x[1][i] = -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------------ rows through shared memory
// One thread per row of the tile; a reader's half of the accumulator's columns passes through registers 64 at a time.
//
// A thread's row is contiguous in memory and its warp's 32 rows are not, so values go through shared memory: every thread
// leaves 128 bytes of its row there (16-byte chunk k at place k ^ (row % 8), so that neither side meets a bank twice), and
// eight threads at a time write one row's 128 bytes.  Written straight from registers, 16 bytes to each of 32 rows at a
// time, the same tile took the probs kernel of 16 x 1024 tokens x 50257 (width 768) 1684 us instead of 1115 us.

// Where a warp's 32 rows go: byte offset of each lane's own row, and which rows are written.
struct Rows {
  char* base;
  int64_t offset;
  unsigned on;
};

__device__ __forceinline__ void stage(uint32_t at, int lane, int chunk, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 128 + ((chunk ^ (lane & 7)) << 4)), "r"(v.x), "r"(v.y),
               "r"(v.z), "r"(v.w)
               : "memory");
}

__device__ __forceinline__ uint4 unstage(uint32_t at, int row, int chunk) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(at + row * 128 + ((chunk ^ (row & 7)) << 4))
               : "memory");
  return v;
}

// Staged rows of 128 bytes to memory, from byte `first` of each row on; chunks at or behind `limit` bytes are left out.
__device__ __forceinline__ void write_staged(const Rows& rows, uint32_t at, int lane, int64_t first, int64_t limit) {
  __syncwarp();
  const int chunk = lane & 7;
  const int64_t byte = first + 16 * chunk;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 4 * i + (lane >> 3);
    const uint4 v = unstage(at, row, chunk);
    const int64_t offset = __shfl_sync(0xffffffffu, rows.offset, row);
    if ((rows.on >> row & 1) && byte < limit) *reinterpret_cast<uint4*>(rows.base + offset + byte) = v;
  }
  __syncwarp();
}

// ------------------------------------------------------------------------------------------------ packing
struct PackParams {
  const __nv_bfloat16* hidden;
  int64_t hidden_stride, hidden_row;
  const void* targets;
  int64_t target_stride;
  bool wide, hidden_vec, d_hidden_vec;
  int n_tokens, vocab, width, rows_pad, row_tile, packed_row;
  __nv_bfloat16* packed;
  int *count, *target, *token_of;
  float* token_loss;
  int64_t token_loss_stride;
  Out d_hidden;             // p NULL: none
  Control* control;
};

// Per token, [replica][n_tokens] with a stride between replicas; p NULL: not wanted, or not given.
template <typename T>
struct PerToken {
  T* p;
  int64_t stride;
  __device__ __forceinline__ T& at(int r, int64_t t) const { return p[r * stride + t]; }
};

constexpr int kNoFloor = (int)0x807fffffu;         // -inf, as an integer of the same order

// What hdet_token_scores writes.
struct ScoreOut {
  PerToken<float> logprob, entropy, lse, top_logprob;   // the last with n_top values a token
  PerToken<int> top_ids;
  int n_top;
  int* floor;               // where packing leaves kNoFloor for every row, or NULL
  __device__ __forceinline__ void padding(int r, int64_t t) const {
    if (logprob.p) logprob.at(r, t) = 0.0f;
    if (entropy.p) entropy.at(r, t) = 0.0f;
    if (lse.p) lse.at(r, t) = 0.0f;
    for (int k = 0; k < n_top; ++k) {
      top_ids.at(r, t * n_top + k) = -1;
      if (top_logprob.p) top_logprob.at(r, t * n_top + k) = 0.0f;
    }
  }
};

// What hdet_token_scores_grad is given: with a and b the gradients of a token's log probability and entropy H, and lp = z - lse the
// logarithms of the probabilities p,  G = a (onehot - p) - b p (lp + H).
//
// Where one class has nearly all of the probability, its lp and H are both near zero, and lp from fp32 logits and an fp32 lse has none of its digits
// left: of d_entropy alone such rows' gradients were 5 to 10 % off at 1 - p of 1e-8 to 1e-12, and up to 2e6 times their value where the logits are
// formed in another order than before.  A row of G adds up to nothing, so that class's entry is less the sum of the others, none of which is
// near zero in that way.  Rows with an entropy below kCertainEntropy are treated so: they have a class
// with a probability of at least exp(-0.25) = 0.78.  Where that is the given token nothing is to do, its own logarithm being given.
constexpr float kCertainEntropy = 0.25f;
constexpr float kLikely = -0.6931472f;             // a class with a larger lp is that class: no other has more than exp(-1.5)

struct ScoreGiven {
  PerToken<const float> lse, logprob, entropy, d_logprob, d_entropy;
  RowNorm* norm;
  int* certain;             // per replica: so many rows are such rows; they are packed before the others.  NULL without d_entropy
  int* likely;              // per row: the class, -1 until it is found
  __device__ __forceinline__ bool is_certain(int r, int64_t t) const {
    if (!certain) return false;
    const float b = d_entropy.at(r, t), h = entropy.at(r, t), lp = logprob.p ? logprob.at(r, t) : -INFINITY;
    return (b != 0.0f) & (h < kCertainEntropy) & !(lp > kLikely);      // (no branch, so that the loads go together)
  }
  __device__ __forceinline__ void row(int64_t row, int r, int64_t t) const {
    const float a = d_logprob.p ? d_logprob.at(r, t) : 0.0f, b = d_entropy.p ? d_entropy.at(r, t) : 0.0f;
    const float h = entropy.p && d_entropy.p ? entropy.at(r, t) : 0.0f, lp = logprob.p ? logprob.at(r, t) : -INFINITY;
    const float p = expf(lp);
    // 1 - p of a likely target from its logarithm, not as a difference
    norm[row] = RowNorm{lse.at(r, t), fmaf(b, h, a), -a * expm1f(lp) - (p > 0.0f ? b * p * (lp + h) : 0.0f), b};
    if (likely) likely[row] = -1;
  }
};

enum PackFor { kPackLoss, kPackScores, kPackGiven };

constexpr int kPackBlocks = 256;   // blocks per replica, about: more would count the targets too often

// The target of a token, -1 for padding.
__device__ __forceinline__ int target_of(const PackParams& p, int r, int t) {
  if (!p.targets) return 0;                      // no targets: every token counts
  const int64_t at = r * p.target_stride + t;
  if (p.wide) {
    const long long v = static_cast<const long long*>(p.targets)[at];
    return v >= 0 && v < p.vocab ? (int)v : -1;
  }
  const int v = static_cast<const int*>(p.targets)[at];
  return v >= 0 && v < p.vocab ? v : -1;
}

// Moves the hidden states of counted tokens together, `rows` tokens a block (a multiple of 8: one a warp at a time).  Every
// block counts the targets before its own (and all of them) itself: that is 4 bytes a token from L2 instead of a launch of its
// own for the offsets.
template <PackFor FOR, typename More>
__global__ void __launch_bounds__(256) pack_kernel(const PackParams p, int rows, const More more) {
  constexpr bool kTwo = FOR == kPackGiven;         // rows of one kind before those of the other
  __shared__ int s_before[8], s_all[8], s_before_first[8], s_all_first[8];
  const int r = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = (int)blockIdx.x * rows, t1 = min(t0 + rows, p.n_tokens);
  let_next_start();
  wait_for_previous();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.control->done[r] = 0;
    if (r == 0) p.control->status = p.control->ticket = 0;
  }
  const auto is_first = [&](int t) {
    if constexpr (kTwo) return more.is_certain(r, t);
    else return false;
  };
  int before = 0, all = 0, before_first = 0, all_first = 0;        // counted tokens, and those of the first kind among them
#pragma unroll 4
  for (int t = threadIdx.x; t < p.n_tokens; t += 256) {
    const int one = target_of(p, r, t) >= 0;
    all += one;
    before += t < t0 ? one : 0;
    if constexpr (kTwo) {
      const int first = is_first(t) ? one : 0;
      all_first += first;
      before_first += t < t0 ? first : 0;
    }
  }
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) { s_before[warp] = before; s_all[warp] = all; }
  if constexpr (kTwo) {
    before_first = __reduce_add_sync(0xffffffffu, before_first);
    all_first = __reduce_add_sync(0xffffffffu, all_first);
    if (lane == 0) { s_before_first[warp] = before_first; s_all_first[warp] = all_first; }
  }
  __syncthreads();
  before = all = before_first = all_first = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    before += s_before[w];
    all += s_all[w];
    if constexpr (kTwo) {
      before_first += s_before_first[w];
      all_first += s_all_first[w];
    }
  }
  before += all_first - before_first;              // the place of the block's first token of the second kind
  const int64_t base = (int64_t)r * p.rows_pad;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.count[r] = all;
    if constexpr (kTwo) {
      if (more.certain) more.certain[r] = all_first;
    }
  }
  // 32 tokens at a time: every warp finds out where they go, and moves every eighth
  for (int first = t0; first < t1; first += 32) {
    const int mine = first + lane;
    const int y = mine < t1 ? target_of(p, r, mine) : -1;
    const unsigned counted = __ballot_sync(0xffffffffu, y >= 0), below = (1u << lane) - 1;
    const unsigned first_kind = kTwo ? __ballot_sync(0xffffffffu, y >= 0 && is_first(mine)) : 0u;
    const int place = first_kind >> lane & 1 ? before_first + __popc(first_kind & below) : before + __popc(counted & ~first_kind & below);
    before += __popc(counted & ~first_kind);
    before_first += __popc(first_kind);
    if (warp == 0 && mine < t1) {
      if (y >= 0) {
        p.target[base + place] = FOR == kPackLoss || p.targets ? y : -1;
        p.token_of[base + place] = mine;
        if constexpr (FOR == kPackScores) {
          if (more.floor) more.floor[base + place] = kNoFloor;
        }
        if constexpr (FOR == kPackGiven) more.row(base + place, r, mine);
      } else if constexpr (FOR == kPackScores) {
        more.padding(r, mine);
      } else if (p.token_loss) {
        p.token_loss[r * p.token_loss_stride + mine] = 0.0f;
      }
    }
    for (int i = warp; i < 32 && first + i < t1; i += 8) {
      const int to = __shfl_sync(0xffffffffu, place, i);
      const int64_t t = first + i;
      if (counted >> i & 1) {
        const __nv_bfloat16* from = p.hidden + r * p.hidden_stride + t * p.hidden_row;
        __nv_bfloat16* dst = p.packed + (base + to) * p.packed_row;
        if (p.hidden_vec) {
#pragma unroll 4
          for (int c = lane * 8; c < p.width; c += 256)
            *reinterpret_cast<uint4*>(dst + c) = *reinterpret_cast<const uint4*>(from + c);
        } else {
#pragma unroll 4
          for (int c = lane; c < p.width; c += 32) dst[c] = from[c];
        }
      } else if (p.d_hidden.p) {
        const int64_t at = r * p.d_hidden.stride + t * p.d_hidden.row;
        const int size = p.d_hidden.f32 ? 4 : 2;
        char* dst = static_cast<char*>(p.d_hidden.p) + at * size;
        if (p.d_hidden_vec) {
          for (int b = lane * 16; b < p.width * size; b += 512) *reinterpret_cast<uint4*>(dst + b) = make_uint4(0, 0, 0, 0);
        } else {
          for (int c = lane; c < p.width; c += 32) {
            if (p.d_hidden.f32) reinterpret_cast<float*>(dst)[c] = 0.0f;
            else reinterpret_cast<__nv_bfloat16*>(dst)[c] = __float2bfloat16_rn(0.0f);
          }
        }
      }
    }
  }
  // rows behind the last counted token, up to the tile's end: zeros, since a product sums over them
  const int end = min(p.rows_pad, (all + p.row_tile - 1) / p.row_tile * p.row_tile);
  for (int row = all + (int)blockIdx.x * 8 + warp; row < end; row += (int)gridDim.x * 8) {
    if (lane == 0) {
      p.target[base + row] = -1;
      p.token_of[base + row] = 0;
      if constexpr (FOR == kPackScores) {
        if (more.floor) more.floor[base + row] = kNoFloor;
      }
    }
    __nv_bfloat16* dst = p.packed + (base + row) * p.packed_row;
    for (int c = lane * 8; c < p.packed_row; c += 256) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0, 0, 0, 0);
  }
}

// A table whose rows cannot be copied as boxes (odd width, stride or address) is laid out once in the workspace, in accesses
// of the largest T that its rows start and end on.  14 tables of 20474 x 996 (8-byte accesses) take 320 us, of 20474 x 997
// (2-byte ones) 460: a width that is a multiple of 8 needs none of it.
template <typename T>
__global__ void __launch_bounds__(256) pack_table_kernel(const __nv_bfloat16* table, int64_t stride, int64_t row, int vocab,
                                                         int width, int packed_row, __nv_bfloat16* packed) {
  const int v = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  let_next_start();
  wait_for_previous();
  if (v >= vocab) return;
  const T* from = reinterpret_cast<const T*>(table + blockIdx.y * stride + v * row);
  T* to = reinterpret_cast<T*>(packed + ((int64_t)blockIdx.y * vocab + v) * packed_row);
#pragma unroll 8
  for (int c = lane; c < width / (int)(sizeof(T) / 2); c += 32) to[c] = from[c];
}

cudaError_t launch_pack_table(const __nv_bfloat16* table, int64_t stride, int64_t row, int vocab, int width, int packed_row, int tables,
                              __nv_bfloat16* packed, cudaStream_t st) {
  const int64_t all = row | stride | width;
  const uintptr_t at = reinterpret_cast<uintptr_t>(table);
  const bool by8 = all % 4 == 0 && at % 8 == 0, by4 = all % 2 == 0 && at % 4 == 0;
  return launch(by8 ? pack_table_kernel<uint2> : by4 ? pack_table_kernel<uint32_t> : pack_table_kernel<uint16_t>,
                dim3((unsigned)div_up(vocab, 8), tables), 256, 0, 1, st, table, stride, row, vocab, width, packed_row, packed);
}

// ------------------------------------------------------------------------------------------------ host side
int fail(int code, const char* who, const char* what) {
  char msg[240];
  snprintf(msg, sizeof msg, "%s: %s", who, what);
  set_handleless_error(msg);
  return code;
}

// The call's own error, which does not stay behind for whoever asks the runtime for its last one next.
int fail_cuda(const char* who, cudaError_t e) {
  cudaGetLastError();
  return fail(HDET_ERR_CUDA, who, cudaGetErrorString(e));
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int elem_size(int dtype) { return dtype == HDET_DTYPE_BF16 ? 2 : 4; }
bool is_float(int dtype) { return dtype == HDET_DTYPE_F32 || dtype == HDET_DTYPE_BF16; }

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

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

constexpr int kMaxDevices = 64;
std::mutex g_mutex;
EncodeTiled g_encode = nullptr;
int g_sms[kMaxDevices];      // SMs of the device, 0 until it is prepared

// Once per process: the driver's tensor-map encoder.  Once per device: the kernels' shared-memory sizes and its SM count.
template <size_t N>
cudaError_t prepare_device(int device, int* sms, const void* const (&kernels)[N], int smem) {
  std::lock_guard<std::mutex> lock(g_mutex);
  if (device >= kMaxDevices) return cudaErrorInvalidDevice;
  if (!g_encode) {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (found != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
    g_encode = reinterpret_cast<EncodeTiled>(f);
  }
  if (g_sms[device]) {
    *sms = g_sms[device];
    return cudaSuccess;
  }
  for (const void* k : kernels) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) g_sms[device] = *sms;
  return e;
}

// [z][y][x] bf16, x contiguous, copied in boxes of 64 x 64; what lies outside reads as zero.
bool encode(CUtensorMap* map, const void* base, int64_t x, int64_t y, int64_t z, int64_t y_stride, int64_t z_stride) {
  const cuuint64_t dims[3] = {(cuuint64_t)x, (cuuint64_t)y, (cuuint64_t)z};
  const cuuint64_t strides[2] = {(cuuint64_t)y_stride * 2, (cuuint64_t)z_stride * 2};
  const cuuint32_t box[3] = {64, 64, 1}, step[3] = {1, 1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace hdet
