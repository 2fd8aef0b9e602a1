// Exact attention, backward: the probabilities are taken again from the row log-sum-exp,
//   P = exp2(s2 q.k + bias - c),  c = log2(e) lse,   dP = dY.v,   D = dY.y,   dS = P (dP - D),
//   dq = scale sum_j dS k,   dk = scale sum_i dS q,   dv = sum_i P dy,   dT[c] = sum of dS in bucket c.
// Two kernels, each summing over its own loop, so that every sum has a fixed order and no result
// depends on the order of atomics: k_exact_dq (per query rows; also D and the bias gradient) and
// k_exact_dkv (per keys, over the query heads that share them). That takes S and dP twice: seven
// products for the five that the formulas need.
#include "exact_device.h"

namespace mca {
namespace {

template <typename T> constexpr int kBwdStages = ExFmt<T>::ES == 2 ? 3 : 2;
template <typename T> constexpr int kDqLds = kExWaves * kBwdStages<T> * 2 * tile_bytes<T>();
template <typename T> constexpr int kDkvStage = 2 * tile_bytes<T>() + 256;  // Q, dY, 32 row statistics
template <typename T> constexpr int kDkvLds = kExWaves * kBwdStages<T> * kDkvStage<T>;
constexpr int kYS = kDHead + 4;  // row pitch of the sums that the waves of a block join in LDS

// Eight consecutive values of a row to `o`.
template <typename T>
__device__ __forceinline__ void ex_store8(T* o, const float (&y)[8]) {
  if constexpr (ExFmt<T>::ES == 2) {
    *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                                              pack_bf16x2(y[6], y[7]));
  } else {
    reinterpret_cast<float4*>(o)[0] = make_float4(y[0], y[1], y[2], y[3]);
    reinterpret_cast<float4*>(o)[1] = make_float4(y[4], y[5], y[6], y[7]);
  }
}
__device__ __forceinline__ void ex_put_sums(float* ys, const f32x16_t (&y)[2], int row, int hf) {
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<float4*>(ys + row * kYS + 32 * cc + 8 * (r >> 2) + 4 * hf) =
          make_float4(y[cc][r], y[cc][r + 1], y[cc][r + 2], y[cc][r + 3]);
}
__device__ __forceinline__ void ex_join_sums(float (&o)[8], const float* ys, int row, int col, float scale) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = ys[row * kYS + col + e];
#pragma unroll
    for (int k = 1; k < kExWaves; ++k) v += ys[(k * 32 + row) * kYS + col + e];
    o[e] = v * scale;
  }
}

// ------------------------------------------------------------------ dQ
// Blocks of 32 (query, head) rows whose key tiles the four waves share, as k_exact_rows. S^T = K Q^T
// and dP^T = V dY^T: the row's c and D are one value per lane, and dS feeds dQ^T = K^T dS^T.
//
// The bias gradient: a pair's dS belongs to entry rel = j - p, and in one register of a half wave the
// 32 lanes (one query position each, or another head) hold 32 different entries. Every half wave
// has an array of its own in LDS, so that no two lanes add to one entry in one instruction and the
// sums have a fixed order; a tile whose pairs all lie D or further away is summed per lane in a
// register and added to entries of the far side that no other lane uses.
template <typename T, bool BIAS>
__global__ __launch_bounds__(kExThreads) void k_exact_dq(ExactParams p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int ES = ExFmt<T>::ES, ST = kBwdStages<T>, TB = tile_bytes<T>();
  const int n = 2 * p.D + 129;
  float* tb = reinterpret_cast<float*>(smem + kDqLds<T>);  // [Gp][n]
  float* dg = tb + p.Gp * n;                               // [wave][half][Gp][n]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5;
  const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp;
  int bid = blockIdx.x;
  const int vt = bid % nvt;
  bid /= nvt;
  const int hx = bid % Hx, b = bid / Hx;
  const ExRow0 br = ex_batch_row(p, b);
  const int hk = hx * p.Gp / p.G;

  const int v = vt * 32 + c, i = v / p.Gp, g = v % p.Gp, head = hx * p.Gp + g;
  const bool live = i < br.qlen;
  const int imin = vt * 32 / p.Gp, imax = min((vt * 32 + 31) / p.Gp, br.qlen - 1);
  const int pmin = br.pos + imin, pmax = br.pos + imax, pend = br.pos + (vt * 32 + 31) / p.Gp;
  const ExTiles tiles = imax >= imin ? ex_key_tiles(p, pmin, pmax, br.klen) : ExTiles{-1, 0, 0};

  const char* Kb = static_cast<const char*>(p.K.data) + (b * p.K.batch + hk * kDHead) * ES;
  const char* Vb = static_cast<const char*>(p.V.data) + (b * p.V.batch + hk * kDHead) * ES;
  const uint32_t lds = lds_addr(smem) + (uint32_t)wave * ST * 2 * TB;
  auto load = [&](int idx, int slot) __attribute__((always_inline)) {  // past the last tile: zeros
    const int k0 = ex_tile_at(tiles, idx) * 32, limit = idx < tiles.n ? br.klen : 0;
    ex_load_tile<T>(ex_rsrc(Kb, p.K.row * ES, k0, limit, ExFmt<T>::RB), (int)p.K.row * ES, lds + slot * 2 * TB, lane);
    ex_load_tile<T>(ex_rsrc(Vb, p.V.row * ES, k0, limit, ExFmt<T>::RB), (int)p.V.row * ES, lds + slot * 2 * TB + TB,
                    lane);
  };
#pragma unroll
  for (int k = 0; k < ST - 1; ++k) load(wave + k * kExWaves, k);

  const int64_t hcol = head * kDHead;
  const char* qrow = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + hcol) * ES;
  const char* yrow = static_cast<const char*>(p.Y.data) + (b * p.Y.batch + i * p.Y.row + hcol) * ES;
  const char* dyrow = static_cast<const char*>(p.dY.data) + (b * p.dY.batch + i * p.dY.row + hcol) * ES;
  const ExRow<T> q = live ? ex_global_row<T>(qrow, hf) : ex_zero_row<T>();
  const ExRow<T> dy = live ? ex_global_row<T>(dyrow, hf) : ex_zero_row<T>();
  float D = 0.f, cr = INFINITY;  // a row without keys, or behind the last query: every P is 0
  if (live) {
    const ExRow<T> y = ex_global_row<T>(yrow, hf);
#pragma unroll
    for (int k = 0; k < ExFmt<T>::NG; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (ES == 2) {
          D = fmaf(__uint_as_float(y.v[k][w] << 16), __uint_as_float(dy.v[k][w] << 16), D);
          D = fmaf(__uint_as_float(y.v[k][w] & 0xffff0000u), __uint_as_float(dy.v[k][w] & 0xffff0000u), D);
        } else {
          D = fmaf(__uint_as_float(y.v[k][w]), __uint_as_float(dy.v[k][w]), D);
        }
      }
    const float lse = p.lse[((int64_t)b * p.H + head) * p.nq + i];
    cr = lse == -INFINITY ? INFINITY : lse * kLog2e;
  }
  D += ex_other_half(D);
  if (wave == 0 && hf == 0 && i < p.nq) p.rowstat[((int64_t)b * p.H + head) * p.nq + i] = make_float2(cr, D);
  const int pos = br.pos + i;
  const ExSpan keys = ex_keys_of(p, pos, br.klen);
  const float* tl = nullptr;
  float* dl = nullptr;
  float far_l = 0.f, far_r = 0.f;
  if constexpr (BIAS) {
    ex_fill_bias<T>(p, tb, hx * p.Gp, p.Gp);
    for (int e = threadIdx.x; e < 2 * kExWaves * p.Gp * n; e += kExThreads) dg[e] = 0.f;
    __syncthreads();
    tl = tb + g * n + p.D + 64;
    dl = dg + ((2 * wave + hf) * p.Gp + g) * n + p.D + 64;
  }
  f32x16_t dq[2] = {ex_zero16(), ex_zero16()};

  int slot = 0;
  for (int idx = wave; idx < tiles.n; idx += kExWaves) {
    wait_lds();  // the tile read last is overwritten by the next loads
    load(idx + (ST - 1) * kExWaves, slot == 0 ? ST - 1 : slot - 1);
    wait_vmcnt<(ST - 1) * 2 * ExFmt<T>::NL>();
    asm volatile("" ::: "memory");
    const char* kt = smem + (wave * ST + slot) * 2 * TB;
    const int k0 = ex_tile_at(tiles, idx) * 32;
    f32x16_t x = ex_rows_product<T>(kt, q, c, hf);
    const f32x16_t dp = ex_rows_product<T>(kt + TB, dy, c, hf);
    int side = 0;
    if constexpr (BIAS) {
      side = ex_bias_side(p, k0, pmin, pend);
      if (side != 0) {
        const float far = tl[side * p.D] - cr;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, far);
      } else {
        const float* at = tl + (k0 + 4 * hf - pos);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, at[(r & 3) + 8 * (r >> 2)] - cr);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, -cr);
    }
    if (!ex_whole(p, pmin, pmax, k0, br.klen)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = ex_in(keys, k0 + 4 * hf + (r & 3) + 8 * (r >> 2)) ? x[r] : -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = ex_exp2(x[r]) * (dp[r] - D);
    if constexpr (BIAS) {
      if (side != 0) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += x[r];
        far_l += side < 0 ? sum : 0.f;
        far_r += side > 0 ? sum : 0.f;
      } else {
        float* at = dl + (k0 + 4 * hf - pos);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          __hip_atomic_fetch_add(at + (r & 3) + 8 * (r >> 2), x[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      }
    }
    ex_cols_product<T>(dq, kt, x, lane);
    slot = slot == ST - 1 ? 0 : slot + 1;
  }
  if constexpr (BIAS) {
    __hip_atomic_fetch_add(dl - p.D - 64 + c, far_l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __hip_atomic_fetch_add(dl + p.D + 64 - c, far_r, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  wait_vmcnt<0>();  // no load is under way into what is written next
  __syncthreads();
  float* ys = reinterpret_cast<float*>(smem);
  ex_put_sums(ys, dq, wave * 32 + c, hf);
  if constexpr (BIAS) {
    for (int e = threadIdx.x; e < p.Gp * n; e += kExThreads) {  // the half waves' arrays
      float t = dg[e];
      for (int k = 1; k < 2 * kExWaves; ++k) t += dg[k * p.Gp * n + e];
      tb[e] = t;
    }
  }
  __syncthreads();
  const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
  const int vr = vt * 32 + row, ir = vr / p.Gp;
  if (ir < p.nq) {
    float o[8];
    ex_join_sums(o, ys, row, col, p.scale);
    ex_store8(static_cast<T*>(p.dQ.data) + b * p.dQ.batch + ir * p.dQ.row + (hx * p.Gp + vr % p.Gp) * kDHead + col, o);
  }
  if constexpr (BIAS) {
    // a bucket's entries are neighbours: distances lo .. hi of its side
    for (int e = threadIdx.x; e < p.Gp * p.buckets; e += kExThreads) {
      const int gg = e / p.buckets, k = e % p.buckets, kk = k % p.side;
      const bool right = k >= p.side;
      const int far = p.D + 64;
      int lo = kk, hi = kk;
      if (kk >= p.E) {
        lo = kk == p.E ? p.E : p.thr[kk - p.E - 1];
        hi = kk - p.E < p.nthr ? p.thr[kk - p.E] - 1 : far;
      }
      int a = right ? max(lo, 1) : -hi, z = right ? hi : -lo;  // rel a .. z
      if (!p.bidirectional && kk == 0) z = far;                // keys behind the query
      const float* t = tb + gg * n + far;
      float sum = 0.f;
      for (int r = a; r <= z; ++r) sum += t[r];
      p.part_bias[((int64_t)(b * nvt + vt) * p.buckets + k) * p.H + hx * p.Gp + gg] = sum;
    }
  }
}

// ------------------------------------------------------------------ dK, dV
// Blocks of 32 keys of a key head; the four waves share the query tiles of all its query heads. S =
// Q K^T and dP = dY V^T with the lane holding a key: P and dS feed dV^T = dY^T P and dK^T = Q^T dS.
// A wave loads its tiles of Q, dY and (c, D) straight into LDS. The blocks behind the last key
// block add up the bias gradient's parts, one (bucket, head) per wave.
template <typename T, bool BIAS>
__global__ __launch_bounds__(kExThreads) void k_exact_dkv(ExactParams p, int heads_at_once) {
  extern __shared__ __align__(16) char smem[];
  constexpr int ES = ExFmt<T>::ES, ST = kBwdStages<T>, TB = tile_bytes<T>(), SB = kDkvStage<T>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nkt = (p.nk + 31) / 32;
  int bid = blockIdx.x;
  if (BIAS && bid >= nkt * p.Hk * p.B) {
    const int e = (bid - nkt * p.Hk * p.B) * kExWaves + wave;  // bucket * H + head
    if (e >= p.buckets * p.H) return;
    float sum = 0.f;
    for (int k = lane; k < p.bias_parts; k += 64) sum += p.part_bias[(int64_t)k * p.buckets * p.H + e];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) {
      if constexpr (ES == 2) static_cast<T*>(p.dtable)[e] = (T)f32_to_bf16_bits(sum);
      else static_cast<T*>(p.dtable)[e] = sum;
    }
    return;
  }
  const int c = lane & 31, hf = lane >> 5, n = 2 * p.D + 129;
  float* tb = reinterpret_cast<float*>(smem + kDkvLds<T>);  // [heads_at_once][n]
  const int kt = bid % nkt;
  bid /= nkt;
  const int hk = bid % p.Hk, b = bid / p.Hk;
  const ExRow0 br = ex_batch_row(p, b);
  const int j = kt * 32 + c, jmax = min(kt * 32 + 31, br.klen - 1);
  const ExTiles tiles = ex_query_tiles(p, br, kt * 32, jmax);
  const ExSpan queries = ex_queries_of(p, br, j);

  const bool live = j < br.klen;
  const char* krow = static_cast<const char*>(p.K.data) + (b * p.K.batch + j * p.K.row + hk * kDHead) * ES;
  const char* vrow = static_cast<const char*>(p.V.data) + (b * p.V.batch + j * p.V.row + hk * kDHead) * ES;
  const ExRow<T> kf = live ? ex_global_row<T>(krow, hf) : ex_zero_row<T>();
  const ExRow<T> vf = live ? ex_global_row<T>(vrow, hf) : ex_zero_row<T>();
  f32x16_t dk[2] = {ex_zero16(), ex_zero16()}, dv[2] = {ex_zero16(), ex_zero16()};
  const uint32_t lds = lds_addr(smem) + (uint32_t)wave * ST * SB;

  for (int g0 = 0; g0 < p.G; g0 += heads_at_once) {
    const int ng = min(heads_at_once, p.G - g0), h0 = hk * p.G + g0;
    if constexpr (BIAS) {
      __syncthreads();
      ex_fill_bias<T>(p, tb, h0, ng);
      __syncthreads();
    }
    const int total = tiles.n * ng;
    auto load = [&](int idx, int slot) __attribute__((always_inline)) {  // past the last tile: zeros
      const int h = h0 + (tiles.n > 0 ? idx / tiles.n : 0);
      const int i0 = (tiles.n > 0 ? ex_tile_at(tiles, idx % tiles.n) : 0) * 32, limit = idx < total ? br.qlen : 0;
      const char* Qb = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + h * kDHead) * ES;
      const char* Yb = static_cast<const char*>(p.dY.data) + (b * p.dY.batch + h * kDHead) * ES;
      const uint32_t to = lds + slot * SB;
      ex_load_tile<T>(ex_rsrc(Qb, p.Q.row * ES, i0, limit, ExFmt<T>::RB), (int)p.Q.row * ES, to, lane);
      ex_load_tile<T>(ex_rsrc(Yb, p.dY.row * ES, i0, limit, ExFmt<T>::RB), (int)p.dY.row * ES, to + TB, lane);
      ex_load_lds4(ex_rsrc(reinterpret_cast<const char*>(p.rowstat + ((int64_t)b * p.H + h) * p.nq), 8, i0, limit, 8),
                   lane * 4, to + 2 * TB);
    };
#pragma unroll
    for (int k = 0; k < ST - 1; ++k) load(wave + k * kExWaves, k);
    int slot = 0;
    for (int idx = wave; idx < total; idx += kExWaves) {
      wait_lds();  // the tile read last is overwritten by the next loads
      load(idx + (ST - 1) * kExWaves, slot == 0 ? ST - 1 : slot - 1);
      wait_vmcnt<(ST - 1) * (2 * ExFmt<T>::NL + 1)>();
      asm volatile("" ::: "memory");
      const char* qt = smem + (wave * ST + slot) * SB;
      const float* stat = reinterpret_cast<const float*>(qt + 2 * TB);
      const int i0 = ex_tile_at(tiles, idx % tiles.n) * 32, p0 = br.pos + i0;
      f32x16_t x = ex_rows_product<T>(qt, kf, c, hf);
      f32x16_t ds = ex_rows_product<T>(qt + TB, vf, c, hf);
      float cr[16], D[16];
#pragma unroll
      for (int k = 0; k < 8; ++k) {  // rows 8 (k / 2) + 4 hf + 2 (k % 2), + 1
        const float4 t = *reinterpret_cast<const float4*>(stat + 2 * (8 * (k >> 1) + 4 * hf + 2 * (k & 1)));
        cr[2 * k] = t.x, D[2 * k] = t.y, cr[2 * k + 1] = t.z, D[2 * k + 1] = t.w;
      }
      if constexpr (BIAS) {
        const float* tl = tb + (idx / tiles.n) * n + p.D + 64;
        const int side = ex_bias_side(p, kt * 32, p0, p0 + 31);
        if (side != 0) {
          const float far = tl[side * p.D];
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, far - cr[r]);
        } else {
          const float* at = tl + (j - p0 - 4 * hf);
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, at[-((r & 3) + 8 * (r >> 2))] - cr[r]);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, -cr[r]);
      }
      // (the sums of keys past the last one are not stored)
      if (i0 + 32 > br.qlen || !ex_whole(p, p0, p0 + 31, kt * 32, 0x7fffffff)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = ex_in(queries, i0 + 4 * hf + (r & 3) + 8 * (r >> 2)) ? x[r] : -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = ex_exp2(x[r]);
        ds[r] = x[r] * (ds[r] - D[r]);
      }
      ex_cols_product<T>(dv, qt + TB, x, lane);
      ex_cols_product<T>(dk, qt, ds, lane);
      slot = slot == ST - 1 ? 0 : slot + 1;
    }
    wait_vmcnt<0>();
  }
  __syncthreads();
  float* ys = reinterpret_cast<float*>(smem);
  ex_put_sums(ys, dk, wave * 32 + c, hf);
  ex_put_sums(ys + kExWaves * 32 * kYS, dv, wave * 32 + c, hf);
  __syncthreads();
  const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8, jr = kt * 32 + row;
  if (jr >= p.nk) return;
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (jr < br.klen) ex_join_sums(o, ys, row, col, p.scale);
  ex_store8(static_cast<T*>(p.dK.data) + b * p.dK.batch + jr * p.dK.row + hk * kDHead + col, o);
  if (jr < br.klen) ex_join_sums(o, ys + kExWaves * 32 * kYS, row, col, 1.f);
  ex_store8(static_cast<T*>(p.dV.data) + b * p.dV.batch + jr * p.dV.row + hk * kDHead + col, o);
}

template <typename K>
hipError_t set_lds(K kernel, size_t lds) {
  return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

template <typename T, bool BIAS>
hipError_t launch_backward(const ExactParams& p, hipStream_t s) {
  const size_t entries = BIAS ? (size_t)exact_bias_entries(p.D) : 0;
  const size_t dq_lds = kDqLds<T> + entries * p.Gp * (1 + 2 * kExWaves) * 4;
  hipError_t e = set_lds(k_exact_dq<T, BIAS>, dq_lds);
  if (e != hipSuccess) return e;
  const int64_t rows = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B;
  hipLaunchKernelGGL((k_exact_dq<T, BIAS>), dim3((unsigned)rows), dim3(kExThreads), dq_lds, s, p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  // heads whose bias tables fit beside the tiles at once
  const int at_once = BIAS ? (int)((163840 - kDkvLds<T>) / (entries * 4)) : p.G;
  const int heads = at_once < p.G ? at_once : p.G;
  const size_t dkv_lds = kDkvLds<T> + entries * heads * 4;
  if ((e = set_lds(k_exact_dkv<T, BIAS>, dkv_lds)) != hipSuccess) return e;
  const int64_t blocks = (int64_t)((p.nk + 31) / 32) * p.Hk * p.B + (BIAS ? (p.buckets * p.H + kExWaves - 1) / kExWaves : 0);
  hipLaunchKernelGGL((k_exact_dkv<T, BIAS>), dim3((unsigned)blocks), dim3(kExThreads), dkv_lds, s, p, heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_exact_backward(const ExactParams& p, hipStream_t s) {
  if (p.bf16) return p.table ? launch_backward<uint16_t, true>(p, s) : launch_backward<uint16_t, false>(p, s);
  return p.table ? launch_backward<float, true>(p, s) : launch_backward<float, false>(p, s);
}

}  // namespace mca
