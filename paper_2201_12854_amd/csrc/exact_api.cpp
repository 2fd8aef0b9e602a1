// C ABI of exact attention: argument checks, the buckets' borders, workspace layout, launches.
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "exact.h"
#include "mca_kernels.h"
#include "mca_status.h"

namespace {

using mca::align256;
using mca::aligned16;
using mca::ExactParams;
using mca::fail;
using mca::ok;

constexpr int64_t kMaxLen = int64_t(1) << 24;
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;  // of 256 threads in one launch
constexpr int64_t kMaxPitch = int64_t(1) << 25;         // bytes from row to row

// ------------------------------------------------------------------ buckets
// A product of small factors, exactly: base 2^32, at most 64 + 64 factors of 9 bits.
struct Big {
  uint32_t w[40] = {1};
  void mul(uint32_t f, int times) {
    for (; times > 0; --times) {
      uint64_t c = 0;
      for (uint32_t& x : w) {
        c += (uint64_t)x * f;
        x = (uint32_t)c;
        c >>= 32;
      }
    }
  }
  bool below(const Big& o) const {
    for (int i = 39; i >= 0; --i)
      if (w[i] != o.w[i]) return w[i] < o.w[i];
    return false;
  }
};

mca_status check_buckets(int32_t buckets, int32_t max_distance, int32_t bidirectional) {
  if (bidirectional != 0 && bidirectional != 1) return fail(MCA_ERR_INVALID_ARGUMENT, "bidirectional must be 0 or 1");
  const int least = bidirectional ? 4 : 2;
  if (buckets < least || buckets > mca::kMaxBuckets || (bidirectional && buckets % 2))
    return fail(MCA_ERR_INVALID_ARGUMENT, "bias buckets must be %s%d..%d (got %d)", bidirectional ? "an even number in " : "",
                least, mca::kMaxBuckets, buckets);
  const int e = (bidirectional ? buckets / 2 : buckets) / 2;
  if (max_distance <= e || max_distance > mca::kMaxBiasDistance)
    return fail(MCA_ERR_INVALID_ARGUMENT, "bias max distance must be in %d..%d (got %d)", e + 1, mca::kMaxBiasDistance,
                max_distance);
  return MCA_OK;
}

// thr[k - 1], 0 < k < m: the smallest d with d >= E (D / E)^(k / m), that is d^m E^k >= E^m D^k.
void set_buckets(ExactParams& p, int32_t buckets, int32_t max_distance, int32_t bidirectional) {
  p.buckets = buckets;
  p.bidirectional = bidirectional;
  p.side = bidirectional ? buckets / 2 : buckets;
  p.E = p.side / 2;
  p.D = max_distance;
  const int m = p.side - p.E;
  p.nthr = m - 1;
  const long double ratio = std::pow((long double)p.D / p.E, 1.0L / m);
  long double t = p.E;
  for (int k = 1; k < m; ++k) {
    t *= ratio;
    const long double near = std::nearbyint(t);
    int d = (int)std::ceil(t);
    if (std::fabs(t - near) < 1e-9L * t) {  // on a border, or too close to it for t to tell
      Big a, b;
      a.mul((uint32_t)near, m);
      a.mul((uint32_t)p.E, k);
      b.mul((uint32_t)p.E, m);
      b.mul((uint32_t)p.D, k);
      d = (int)near + (a.below(b) ? 1 : 0);
    }
    p.thr[k - 1] = d;
  }
}

// ------------------------------------------------------------------ checks
mca_status check_exact(const mca_exact_desc* d) {
  if (!d) return fail(MCA_ERR_INVALID_ARGUMENT, "desc is NULL");
  if (d->batch < 1 || d->q_len < 1 || d->kv_len < 1 || d->heads < 1 || d->kv_heads < 1 || d->d_head < 1)
    return fail(MCA_ERR_INVALID_ARGUMENT, "batch, q_len, kv_len, heads, kv_heads and d_head must be >= 1");
  if (d->dtype != MCA_F32 && d->dtype != MCA_BF16)
    return fail(MCA_ERR_INVALID_ARGUMENT, "dtype %d is not MCA_F32 or MCA_BF16", d->dtype);
  if (d->heads > 1024 || d->heads % d->kv_heads)
    return fail(MCA_ERR_INVALID_ARGUMENT, "heads must be at most 1024 and a multiple of kv_heads (got %lld and %lld)",
                (long long)d->heads, (long long)d->kv_heads);
  if (d->batch > kMaxLen || d->q_len > kMaxLen || d->kv_len > kMaxLen)
    return fail(MCA_ERR_INVALID_ARGUMENT, "batch, q_len and kv_len must be at most 2^24");
  if (d->causal != 0 && d->causal != 1) return fail(MCA_ERR_INVALID_ARGUMENT, "causal must be 0 or 1");
  if (d->window < 0 || d->window % 2 != 0 || d->window > (int64_t(1) << 25))
    return fail(MCA_ERR_INVALID_ARGUMENT, "window must be 0 or an even number of keys in 2..2^25 (got %lld)",
                (long long)d->window);
  // least: the bfloat16 backward pass starts its sums at -lse / scale, |lse| up to 2^22
  if (!(d->scale >= 0x1p-100) || !std::isfinite((float)(d->scale * 1.4426950408889634)))
    return fail(MCA_ERR_INVALID_ARGUMENT, "scale must be at least 2^-100 and finite in float32 (got %g)", d->scale);
  if (d->reserved != 0) return fail(MCA_ERR_INVALID_ARGUMENT, "reserved must be 0");
  for (const int32_t* v : {d->q_lens, d->kv_lens, d->q_pos})
    if (reinterpret_cast<uintptr_t>(v) & 3u) return fail(MCA_ERR_INVALID_ARGUMENT, "q_lens, kv_lens and q_pos must be 4-byte aligned");
  if (d->bias_table) {
    if (!aligned16(d->bias_table)) return fail(MCA_ERR_INVALID_ARGUMENT, "device pointers must be 16-byte aligned");
    const mca_status st = check_buckets(d->bias_buckets, d->bias_max_distance, d->bias_bidirectional);
    if (st != MCA_OK) return st;
  }
  if (d->d_head != 64) return fail(MCA_ERR_UNSUPPORTED, "d_head must be 64 (got %lld)", (long long)d->d_head);
  // every launch of either pass, with the fewest heads side by side (float32: the rows' blocks, an eighth of all at
  // most, and the keys' in one)
  const int64_t q = mca::exact_row_tiles(d->q_len, 1), k = (d->kv_len + 31) / 32;
  if ((q * 8 > kMaxBlocks / d->heads / d->batch) || (k + 1 > (kMaxBlocks / 8 * 7 - mca::kMaxBuckets * 1024) / d->kv_heads / d->batch))
    return fail(MCA_ERR_INVALID_ARGUMENT, "batch * heads * length too large for one launch");
  return MCA_OK;
}

// The rows of a [B, n, width] tensor; `out`: they must not overlap.
mca_status check_rows(const mca_rows* t, const char* name, int64_t B, int64_t n, int64_t width, int es, bool out) {
  if (!t || !t->data) return fail(MCA_ERR_INVALID_ARGUMENT, "%s must not be NULL", name);
  if (!aligned16(t->data)) return fail(MCA_ERR_INVALID_ARGUMENT, "%s: device pointers must be 16-byte aligned", name);
  const int64_t unit = 16 / es, b = t->batch_stride, r = t->row_stride;
  if (r < width || r >= kMaxPitch / es || r % unit)
    return fail(MCA_ERR_INVALID_ARGUMENT, "%s: row_stride must be a multiple of 16 bytes, at least the row's %lld elements and below 2^25 bytes (got %lld)",
                name, (long long)width, (long long)r);
  if (b < 0 || b % unit || b > (int64_t(1) << 48))
    return fail(MCA_ERR_INVALID_ARGUMENT, "%s: batch_stride must be a multiple of 16 bytes in 0..2^48 (got %lld)", name, (long long)b);
  if (out && B > 1 && n > 0 && b < (n - 1) * r + width && (b < width || r < (B - 1) * b + width))
    return fail(MCA_ERR_INVALID_ARGUMENT, "%s: the rows of an output must not overlap", name);
  return MCA_OK;
}

ExactParams params_of(const mca_exact_desc& d, bool backward) {
  ExactParams p;
  std::memset(&p, 0, sizeof p);
  p.B = (int)d.batch;
  p.nq = (int)d.q_len;
  p.nk = (int)d.kv_len;
  p.H = (int)d.heads;
  p.Hk = (int)d.kv_heads;
  p.G = p.H / p.Hk;
  p.causal = d.causal;
  p.window = d.window > 0;
  p.half = (int)(d.window / 2);
  p.bf16 = d.dtype == MCA_BF16;
  p.scale = (float)d.scale;
  p.s2 = (float)(d.scale * 1.4426950408889634);
  p.q_lens = d.q_lens;
  p.kv_lens = d.kv_lens;
  p.q_pos = d.q_pos;
  p.table = d.bias_table;
  if (p.table) set_buckets(p, d.bias_buckets, d.bias_max_distance, d.bias_bidirectional);
  p.Gp = mca::exact_group(p);
  p.splits = backward ? 1 : mca::exact_splits(p);
  p.kv_splits = backward ? mca::exact_kv_splits(p) : 1;
  p.bias_parts = backward ? mca::exact_bias_parts(p) : 0;
  return p;
}

// Sets p's workspace pointers from `ws` and returns the size.
size_t carve(ExactParams& p, bool backward, char* ws) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* at = ws ? ws + off : nullptr;  // null: only the size is asked for
    off += align256(bytes);
    return at;
  };
  if (backward && mca::exact_backward_small(p)) return 0;
  if (backward) {
    p.rowstat = reinterpret_cast<float*>(take(8 * (size_t)p.B * p.H * p.nq));
    if (p.kv_splits > 1) {
      const size_t rows = 4 * 64 * (size_t)p.kv_splits * p.B * p.nk * p.Hk;
      p.part_dk = reinterpret_cast<float*>(take(rows));
      p.part_dv = reinterpret_cast<float*>(take(rows));
    }
    if (p.table) p.part_bias = reinterpret_cast<float*>(take(4 * (size_t)p.bias_parts * p.buckets * p.H));
  } else if (p.splits > 1) {
    const size_t rows = (size_t)p.splits * p.B * (p.H / p.Gp) * mca::exact_row_tiles(p.nq, p.Gp) * 32;
    p.part_y = reinterpret_cast<float*>(take(rows * 64 * 4));
    p.part_ml = reinterpret_cast<float2*>(take(rows * sizeof(float2)));
  }
  return off;
}

mca_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return MCA_OK;
  if (!ws) return fail(MCA_ERR_INVALID_ARGUMENT, "workspace must not be NULL (%zu bytes)", need);
  if (!aligned16(ws)) return fail(MCA_ERR_INVALID_ARGUMENT, "device pointers must be 16-byte aligned");
  if (bytes < need) return fail(MCA_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, needs %zu", bytes, need);
  return MCA_OK;
}

// Results that begin where another operand does: in-place calls, one buffer for two gradients. (Overlaps in general
// are not looked for: gradients may be interleaved slices of one tensor.)
mca_status check_apart(std::initializer_list<const void*> in, std::initializer_list<const void*> out) {
  for (const void* const* o = out.begin(); o != out.end(); ++o) {
    for (const void* x : in)
      if (*o && x == *o) return fail(MCA_ERR_INVALID_ARGUMENT, "a result must not be in an operand's memory");
    for (const void* const* u = out.begin(); u != o; ++u)
      if (*o && *u == *o) return fail(MCA_ERR_INVALID_ARGUMENT, "two results must not be in the same memory");
  }
  return MCA_OK;
}

mca::ExactRows rows_in(const mca_rows* t) { return {t->data, t->batch_stride, t->row_stride}; }
mca::ExactOut rows_out(const mca_rows* t) { return {t->data, t->batch_stride, t->row_stride}; }

}  // namespace

extern "C" {

mca_status mca_relative_buckets(int32_t buckets, int32_t max_distance, int32_t bidirectional, int32_t* out) {
  const mca_status st = check_buckets(buckets, max_distance, bidirectional);
  if (st != MCA_OK) return st;
  if (!out) return fail(MCA_ERR_INVALID_ARGUMENT, "out is NULL");
  ExactParams p;
  set_buckets(p, buckets, max_distance, bidirectional);
  for (int r = -p.D; r <= p.D; ++r) {
    const int d = bidirectional ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
    int n = d;
    if (d >= p.E) {
      n = p.E;
      for (int k = 0; k < p.nthr; ++k) n += p.thr[k] <= d ? 1 : 0;
    }
    out[r + p.D] = n + (bidirectional && r > 0 ? p.side : 0);
  }
  return ok();
}

mca_status mca_exact_workspace_size(const mca_exact_desc* desc, int backward, size_t* bytes) {
  const mca_status st = check_exact(desc);
  if (st != MCA_OK) return st;
  if (!bytes) return fail(MCA_ERR_INVALID_ARGUMENT, "bytes is NULL");
  ExactParams p = params_of(*desc, backward != 0);
  *bytes = carve(p, backward != 0, nullptr);
  return ok();
}

mca_status mca_exact_attention_forward(const mca_exact_desc* desc, const mca_rows* Q, const mca_rows* K,
                                       const mca_rows* V, const mca_rows* Y, float* lse, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  mca_status st = check_exact(desc);
  if (st != MCA_OK) return st;
  const int es = desc->dtype == MCA_BF16 ? 2 : 4;
  const int64_t B = desc->batch, wq = desc->heads * 64, wk = desc->kv_heads * 64;
  if ((st = check_rows(Q, "Q", B, desc->q_len, wq, es, false)) != MCA_OK) return st;
  if ((st = check_rows(K, "K", B, desc->kv_len, wk, es, false)) != MCA_OK) return st;
  if ((st = check_rows(V, "V", B, desc->kv_len, wk, es, false)) != MCA_OK) return st;
  if ((st = check_rows(Y, "Y", B, desc->q_len, wq, es, true)) != MCA_OK) return st;
  if (!lse || !aligned16(lse)) return fail(MCA_ERR_INVALID_ARGUMENT, "lse must be a 16-byte aligned device pointer");
  ExactParams p = params_of(*desc, false);
  if ((st = check_workspace(workspace, workspace_bytes, carve(p, false, static_cast<char*>(workspace)))) != MCA_OK) return st;
  if ((st = check_apart({Q->data, K->data, V->data, desc->bias_table}, {Y->data, lse, workspace})) != MCA_OK) return st;
  p.Q = rows_in(Q);
  p.K = rows_in(K);
  p.V = rows_in(V);
  p.Yo = rows_out(Y);
  p.lse = lse;
  const hipError_t e = mca::launch_exact_forward(p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(MCA_ERR_HIP, "exact attention forward launch failed: %s", hipGetErrorString(e));
  return ok();
}

mca_status mca_exact_attention_backward(const mca_exact_desc* desc, const mca_rows* dY, const mca_rows* Q,
                                        const mca_rows* K, const mca_rows* V, const mca_rows* Y, const float* lse,
                                        const mca_rows* dQ, const mca_rows* dK, const mca_rows* dV, void* dbias_table,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  mca_status st = check_exact(desc);
  if (st != MCA_OK) return st;
  const int es = desc->dtype == MCA_BF16 ? 2 : 4;
  const int64_t B = desc->batch, nq = desc->q_len, nk = desc->kv_len, wq = desc->heads * 64, wk = desc->kv_heads * 64;
  if ((st = check_rows(dY, "dY", B, nq, wq, es, false)) != MCA_OK) return st;
  if ((st = check_rows(Q, "Q", B, nq, wq, es, false)) != MCA_OK) return st;
  if ((st = check_rows(K, "K", B, nk, wk, es, false)) != MCA_OK) return st;
  if ((st = check_rows(V, "V", B, nk, wk, es, false)) != MCA_OK) return st;
  if ((st = check_rows(Y, "Y", B, nq, wq, es, false)) != MCA_OK) return st;
  if ((st = check_rows(dQ, "dQ", B, nq, wq, es, true)) != MCA_OK) return st;
  if ((st = check_rows(dK, "dK", B, nk, wk, es, true)) != MCA_OK) return st;
  if ((st = check_rows(dV, "dV", B, nk, wk, es, true)) != MCA_OK) return st;
  if (!lse || !aligned16(lse)) return fail(MCA_ERR_INVALID_ARGUMENT, "lse must be a 16-byte aligned device pointer");
  if (!desc->bias_table != !dbias_table)
    return fail(MCA_ERR_INVALID_ARGUMENT, "dbias_table goes with a bias table: both or neither");
  if (!aligned16(dbias_table)) return fail(MCA_ERR_INVALID_ARGUMENT, "device pointers must be 16-byte aligned");
  ExactParams p = params_of(*desc, true);
  if ((st = check_workspace(workspace, workspace_bytes, carve(p, true, static_cast<char*>(workspace)))) != MCA_OK) return st;
  if ((st = check_apart({dY->data, Q->data, K->data, V->data, Y->data, lse, desc->bias_table},
                        {dQ->data, dK->data, dV->data, dbias_table, workspace})) != MCA_OK) return st;
  p.Q = rows_in(Q);
  p.K = rows_in(K);
  p.V = rows_in(V);
  p.Y = rows_in(Y);
  p.dY = rows_in(dY);
  p.dQ = rows_out(dQ);
  p.dK = rows_out(dK);
  p.dV = rows_out(dV);
  p.lse = const_cast<float*>(lse);
  p.dtable = dbias_table;
  const hipError_t e = mca::launch_exact_backward(p, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(MCA_ERR_HIP, "exact attention backward launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // extern "C"
