// Host-side launch interface of the exact attention kernels (internal to libmca).
#pragma once

#include <hip/hip_runtime.h>
#include <atomic>
#include <stddef.h>
#include <stdint.h>

namespace mca {

constexpr int kMaxBuckets = 128;       // rows of the relative bias table
constexpr int kMaxBiasDistance = 256;  // distances from here on share the last bucket

// Rows of a [batch, rows, heads * 64] tensor: strides in elements, heads and columns contiguous.
struct ExactRows {
  const void* data;
  int64_t batch, row;
};
struct ExactOut {
  void* data;
  int64_t batch, row;
};

struct ExactParams {
  int B, nq, nk, H, Hk;
  int G;                      // query heads per key head
  int Gp;                     // heads that the kernels of 32 rows put side by side (1 or G)
  int causal, window, half;   // window: 0 none, else |p - j| <= half, or p = 0, or j = 0
  int bf16;
  float scale, s2;            // s2 = scale log2(e)
  const int32_t *q_lens, *kv_lens, *q_pos;  // [B] or null
  ExactRows Q, K, V, Y, dY;
  ExactOut Yo, dQ, dK, dV;
  float* lse;                 // [B, H, nq], natural logarithm
  // relative bias
  const void* table;          // [buckets, H] or null
  void* dtable;
  int buckets, side;          // side: buckets of one direction (all of them if not bidirectional)
  int bidirectional, E, D;    // distances below E have a bucket each, those from D on the last one
  int nthr;                   // distances from thr[k] on are in bucket E + 1 + k or a later one
  int thr[kMaxBuckets / 2];
  // workspace
  int splits;                 // forward: parts of the keys that blocks of their own take
  float* part_y;              // [splits][rows of 32][64] sums of P V under the part's maximum
  float2* part_ml;            // [splits][rows of 32] that maximum (base-2 units) and the sum of P
  float* rowstat;             // backward: two planes [B, H, nq] that k_exact_dkv starts from: of a row with
                              // c = log2(e) log-sum-exp (infinity without keys) and D = dY . Y, float32
                              // c and D, bf16 -c / s2 and -D (where its accumulators start)
  int kv_splits;              // parts of the query tiles of a key head that blocks of their own take
  float *part_dk, *part_dv;   // [kv_splits][B, nk, Hk, 64]
  float* part_bias;           // [bias_parts][buckets][H]
  int64_t bias_parts;
};

inline int exact_bias_entries(int D) { return 2 * D + 129; }  // rel = j - p in [-D - 64, D + 64]
// Rows (query, head) that the kernels of 32 rows pad to.
inline int64_t exact_row_tiles(int64_t nq, int64_t Gp) { return (nq * Gp + 31) / 32; }

// Calls whose (batch row, head)s fit a block each: bf16, at most so many queries and keys. Without shared key heads
// the backward pass is one launch then, without a workspace.
constexpr int kSmallRows = 128;
inline bool exact_small(const ExactParams& p) { return p.bf16 && !p.table && p.nq <= kSmallRows && p.nk <= kSmallRows; }
inline bool exact_backward_small(const ExactParams& p) { return exact_small(p) && p.G == 1; }
// Rows that such a block has room for, 32 for each of its waves: with fewer waves more blocks are on a CU
// (backward pass, against four always: 128 x 32 tokens, 12 heads, 12.4 and 19.9 us, 64 x 64 14.2 and 17.7, 300 x
// 40, 16 heads, 46 and 73).
__host__ __device__ inline int exact_small_rows(const ExactParams& p) { return ((p.nq > p.nk ? p.nq : p.nk) + 31) / 32 * 32; }

constexpr size_t kMaxLds = 163840;  // of a block: a CU's

// Allows kernel K that much LDS less STATIC of its own, once per device; an error where `lds` is more.
template <auto K, int STATIC = 0>
hipError_t exact_set_lds(size_t lds) {
  static std::atomic<int> allowed[64];
  int dev = 0;
  if (lds > kMaxLds - STATIC) return hipErrorInvalidValue;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (allowed[dev].load(std::memory_order_acquire)) return hipSuccess;
  // idempotent: threads racing here all set the same attribute before any of them launches
  const hipError_t e = hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxLds - STATIC);
  if (e == hipSuccess) allowed[dev].store(1, std::memory_order_release);
  return e;
}

// Whether `tiles` of 32 over four waves are worth splitting into n parts: what that saves in tiles one after
// another, each `unit` times 0.55 us, against the 3 us of the launch that joins them.
inline bool exact_worth(int64_t tiles, int64_t n, int unit) {
  return ((tiles + 3) / 4 - (tiles + 4 * n - 1) / (4 * n)) * unit >= 6;
}
bool exact_eight_waves(int64_t blocks, int64_t tiles);  // of the kernels of 32 rows, for a block's tiles
int exact_splits(const ExactParams& p);
int exact_kv_splits(const ExactParams& p);
int64_t exact_bias_parts(const ExactParams& p);
int exact_group(const ExactParams& p);  // Gp
// Kernels that a call's sizes choose: in blocks of 32 rows (all float32 calls), of a whole short row, of 128 rows, of
// 256. The backward pass for dQ and for dK and dV.
enum class ExactKernel { kRows32, kShort, kRows128, kRows256 };
ExactKernel exact_forward_kernel(const ExactParams& p);
ExactKernel exact_dq_kernel(const ExactParams& p);
ExactKernel exact_dkv_kernel(const ExactParams& p);
hipError_t launch_exact_forward(const ExactParams& p, hipStream_t s);
hipError_t launch_exact_backward(const ExactParams& p, hipStream_t s);

}  // namespace mca
