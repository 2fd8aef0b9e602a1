// Exact attention, backward: the probabilities are taken again from the row log-sum-exp,
//   P = exp2(s2 q.k + bias - c),  c = log2(e) lse,   dP = dY.v,   D = dY.y,   dS = P (dP - D),
//   dq = scale sum_j dS k,   dk = scale sum_i dS q,   dv = sum_i P dy,   dT[c] = sum of dS in bucket c.
// Two parts, each summing over its own loop, so that every sum has a fixed order and no result depends on the
// order of atomics: dQ (per query rows) and dK, dV (per keys, over the query heads that share them; also the bias
// gradient). That takes S and dP twice: seven products for the five that the formulas need. bf16: a launch
// each, as the second needs a D that only the first has (below); up to 128 rows one launch of blocks that
// have both. float32: k_exact_stats, then one launch of both parts' blocks, which fill the card together
// (backward pass, 12 heads, a launch each against this: 2 x 333 tokens 64.3 and 50.4 us, 1 x 128 22.1 and
// 13.9, 8 x 512 225 and 222). k_exact_join_grads adds up what blocks leave in parts.
#include <algorithm>

#include "exact_device.h"
#include "mca_kernels.h"

namespace mca {
namespace {

// ST: tiles in LDS per wave of the blocks of 32 rows, all but one of them on their way: two in bf16, one in
// float32, where two such blocks on a CU cover each other's loads. W: waves of the block.
template <typename T, int ST, int W> constexpr int kDqLds = W * ST * 2 * tile_bytes<T>();
template <typename T> constexpr int kDkvStage = 2 * tile_bytes<T>() + 512;  // Q, dY, two planes of statistics
template <typename T, int ST, int W> constexpr int kDkvLds = W * ST * kDkvStage<T>;
constexpr int kYS = kDHead + 4;  // row pitch of the sums that the waves of a block join in LDS

// Four consecutive values of a row to `o`.
template <typename T>
__device__ __forceinline__ void ex_store4(T* o, float4 y) {
  if constexpr (ExFmt<T>::ES == 2) *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
  else *reinterpret_cast<float4*>(o) = y;
}
__device__ __forceinline__ void ex_put_sums(float* ys, const f32x16_t (&y)[2], int row, int hf) {
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<float4*>(ys + row * kYS + 32 * cc + 8 * (r >> 2) + 4 * hf) =
          make_float4(y[cc][r], y[cc][r + 1], y[cc][r + 2], y[cc][r + 3]);
}
// Four columns of a row, summed over the waves in their order.
template <int W>
__device__ __forceinline__ float4 ex_join_sums(const float* ys, int row, int col, float scale) {
  float4 v = *reinterpret_cast<const float4*>(ys + row * kYS + col);
#pragma unroll
  for (int k = 1; k < W; ++k) {
    const float4 t = *reinterpret_cast<const float4*>(ys + (k * 32 + row) * kYS + col);
    v.x += t.x, v.y += t.y, v.z += t.z, v.w += t.w;
  }
  return make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
}

// c of a row, infinity (every P is 0) for one without keys. P is off by as much as float32 leaves of c, about |c|
// 2^-18 (with the start of S at -c / s2 in bf16); where lse itself is only known to halves, past 2^22, it would be
// anything up to infinity, so such a row (all its biases that large) takes no part either.
__device__ __forceinline__ float ex_row_offset(float lse) { return fabsf(lse) > 0x1p22f ? INFINITY : lse * kLog2e; }
// What k_exact_dkv starts from, bf16.
__device__ __forceinline__ void ex_put_stat(const ExactParams& p, int64_t row, float c, float D) {
  p.rowstat[row] = -c * (1.f / p.s2);
  p.rowstat[(int64_t)p.B * p.H * p.nq + row] = -D;
}
// float32: c and D, 16 lanes a row.
__global__ __launch_bounds__(kExThreads) void k_exact_stats(ExactParams p) {
  const int64_t rows = (int64_t)p.B * p.nq * p.H, e = (int64_t)blockIdx.x * (kExThreads / 16) + (threadIdx.x >> 4);
  if (e >= rows) return;  // (rows of 16 lanes leave together)
  const int h = (int)(e % p.H), i = (int)(e / p.H % p.nq), b = (int)(e / p.H / p.nq);
  const int64_t row = ((int64_t)b * p.H + h) * p.nq + i, col = h * kDHead + 4 * (threadIdx.x & 15);
  float D = 0.f, c = INFINITY;  // as in ex_dq_block
  if (i < ex_batch_row(p, b).qlen) {
    const float4 y = *reinterpret_cast<const float4*>(static_cast<const float*>(p.Y.data) + b * p.Y.batch + i * p.Y.row + col);
    const float4 g = *reinterpret_cast<const float4*>(static_cast<const float*>(p.dY.data) + b * p.dY.batch + i * p.dY.row + col);
    D = fmaf(y.w, g.w, fmaf(y.z, g.z, fmaf(y.y, g.y, y.x * g.x)));
    const float lse = p.lse[row];
    c = ex_row_offset(lse);
  }
  D += dpp_f32<0xB1>(D);
  D += dpp_f32<0x4E>(D);
  D += dpp_f32<0x141>(D);
  D += dpp_f32<0x140>(D);
  if ((threadIdx.x & 15) == 0) {
    p.rowstat[row] = c;
    p.rowstat[(int64_t)p.B * p.H * p.nq + row] = D;
  }
}

// ------------------------------------------------------------------ sums along diagonals
// The bias gradient needs dS summed by rel = j - p, along the diagonals of a tile. In the registers of
// k_exact_dkv a lane is a key and a register a query, so a step to the next query and the next
// key is a step to the next register and lane: sums of the form acc = shift(acc) + x[r], one vector
// instruction per pair with the lane shift in it, collect diagonals. A shift stays within 16 lanes
// and what it pushes out is lost: of a block of 16 keys and 16 queries, shifting up collects the
// diagonals rel < 0, one to a lane, shifting down those of rel >= 0. (Adding every pair to an array with
// LDS atomics took 130 cycles an instruction: 16 x 512 tokens, 12 heads, 306 us for the kernel that had
// it.)
template <int CTRL>
__device__ __forceinline__ float ex_shift(float v) {  // within rows of 16 lanes, zeros shifted in
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float ex_shift_rows(float v) {  // only the rows of 16 lanes in ROWS
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), CTRL,
                                                               ROWS, 0xF, true));
}
template <int ROWS>
__device__ __forceinline__ float ex_rows_only(float v) {  // zeros in the other rows
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xE4, ROWS, 0xF, false));
}
// A wave's sums: dg, an array of entries, and the lower half of the last tile's, in lanes 32 and up. A diagonal of a
// wave's keys passes two tiles of queries, one after the other, so what the next tile has is added in a
// register and every entry is stored once.
struct ExDiag {
  float* dg;
  float pend;
  int at;  // the entry of pend's lane 32, -1: none
};
__device__ __forceinline__ void ex_diag_flush(ExDiag& d, int lane) {
  if (d.at >= 0 && lane >= 32) d.dg[d.at + lane - 32] = d.pend;
  d.at = -1;
}
// Tile x, whose key 0 and query 0 have entry `at`: its diagonals are the entries at - 31 .. at + 31.
__device__ __forceinline__ void ex_diagonals(ExDiag& d, const f32x16_t& x, int at, int lane_) {
  const int lane = ex_opaque(lane_);
  float up[2], down[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {  // queries 16 kb + {0 .. 3, 8 .. 11} + 4 hf
    up[kb] = x[8 * kb];
    down[kb] = x[8 * kb + 7];
  }
#pragma unroll
  for (int r = 1; r < 8; ++r)
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      up[kb] = (r == 4 ? ex_shift<0x115>(up[kb]) : ex_shift<0x111>(up[kb])) + x[8 * kb + r];
      down[kb] = (r == 4 ? ex_shift<0x105>(down[kb]) : ex_shift<0x101>(down[kb])) + x[8 * kb + 7 - r];
    }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    up[kb] = ex_shift_rows<0x111, 0xC>(ex_shift_rows<0x115, 0x3>(up[kb]));  // query 11 + 4 hf to 16
    down[kb] = ex_shift_rows<0x104, 0xC>(down[kb]);                         // query 4 hf to 0
  }
  // Rows of 16 lanes by (query half hf, key half a): up of key half a and queries kb has the 16 entries from
  // 16 (a - kb) - 16 on, down those from 16 (a - kb) on. As rows of entries from -32, -16, 0, 16 on:
  // up[1] and down[0] added over hf are the four rows, and up[0] + down[1] belongs to the middle two.
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(up[1]), __float_as_uint(down[0]), false, false);
  float w = up[0] + down[1];
  w += ex_other_half(w);
  const auto m = __builtin_amdgcn_permlane16_swap(__float_as_uint(w), __float_as_uint(w), false, false);
  float v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  v += ex_rows_only<0x2>(__uint_as_float(m[0])) + ex_rows_only<0x4>(__uint_as_float(m[1]));
  if (d.at != at) {
    ex_diag_flush(d, lane);
    d.pend = 0.f;
  }
  if (lane >= 32) d.dg[at + lane - 32] = v + d.pend;
  d.pend = ex_other_half(v);
  d.at = at - 32;
}
// Takes a wave's sums of a head out as a part of the bias gradient: far tiles' sums per lane (`left`: rel
// <= -D, `right`: rel >= D) and the array, which is left as zeros. A bucket's entries are neighbours; four
// lanes share those of a bucket.
__device__ __forceinline__ void ex_put_buckets(const ExactParams& p, ExDiag& d, int n, float left, float right, int64_t part,
                                               int head, int lane_) {
  const int lane = ex_opaque(lane_);
  float* dg = d.dg;
  ex_diag_flush(d, lane);
  wave_lds_sync();
  left += ex_other_half(left);
  right += ex_other_half(right);
  if (lane < 32) {  // entries of the far sides, one per lane
    dg[lane] += left;
    dg[n - 1 - lane] += right;
  }
  wave_lds_sync();
  const int far = p.D + 64;
  for (int k0 = 0; k0 < p.buckets; k0 += 16) {
    const int k = min(k0 + (lane >> 2), p.buckets - 1), kk = k % p.side;
    const bool ahead = k >= p.side;
    int lo = kk, hi = kk;  // distances
    if (kk >= p.E) {
      lo = kk == p.E ? p.E : p.thr[kk - p.E - 1];
      hi = kk - p.E < p.nthr ? p.thr[kk - p.E] - 1 : far;
    }
    const int a = ahead ? max(lo, 1) : -hi;
    const int z = ahead ? hi : !p.bidirectional && kk == 0 ? far : -lo;  // keys ahead share bucket 0
    float sum = 0.f;
#pragma unroll 8
    for (int r = a + (lane & 3); r <= z; r += 4) sum += dg[far + r];
    sum += dpp_f32<0xB1>(sum);
    sum += dpp_f32<0x4E>(sum);
    if ((lane & 3) == 0 && k0 + (lane >> 2) < p.buckets) p.part_bias[(part * p.buckets + k) * p.H + head] = sum;
  }
  wave_lds_sync();
#pragma unroll 4
  for (int e = lane; e < n; e += 64) dg[e] = 0.f;
  wave_lds_sync();
}
template <typename T>
__device__ __forceinline__ float ex_sum16(const T& x) {
  float s = x[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) s += x[r];
  return s;
}

// D plus the lane's part of a . b.
template <typename T>
__device__ __forceinline__ float ex_row_dot(const ExRow<T>& a, const ExRow<T>& b, float D) {
#pragma unroll
  for (int k = 0; k < ExFmt<T>::NG; ++k)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (ExFmt<T>::ES == 2) {
        D = fmaf(__uint_as_float(a.v[k][w] << 16), __uint_as_float(b.v[k][w] << 16), D);
        D = fmaf(__uint_as_float(a.v[k][w] & 0xffff0000u), __uint_as_float(b.v[k][w] & 0xffff0000u), D);
      } else {
        D = fmaf(__uint_as_float(a.v[k][w]), __uint_as_float(b.v[k][w]), D);
      }
    }
  return D;
}

// FEW of the kernels below: P and dS are multiplied to more than the type's bits (ex_cols_product). By the lengths
// alone, so that a row's precision does not depend on how many there are: up to 32 queries or keys, a tile, whose
// roundings do not average out.
bool few(const ExactParams& p) { return p.bf16 && std::min(p.nq, p.nk) <= 32; }

// ------------------------------------------------------------------ dQ
// Blocks of 32 (query, head) rows whose key tiles the waves share, as k_exact_rows. S^T = K Q^T
// and dP^T = V dY^T: the row's c and D are one value per lane, and dS feeds dQ^T = K^T dS^T.
//
//
// dS cancels where attention is sharp, and in bf16 D' = dY . Y of the rounded Y (whose P were rounded too)
// is not exact enough then: the gradients would lose as much as by all other roundings (8 x 300 tokens,
// logits of standard deviation 2: dQ off by 3.8e-3 of its norm; 2.4e-3 with the exact D, 1.7e-3 of it the
// result's own rounding). The exact D comes out of the sums: sum_j dS'_ij = D - D', so sum_j P_ij k_j is
// summed beside dq, dq = scale (sum_j dS' k - (D - D') sum_j P k), and k_exact_dkv gets D. What D - D' is
// comes from large P, and is multiplied by them: the kernel of 64-row tiles leaves half tiles out of sum_j P k
// whose P are all at most kSmallP (at 4 x 4096 tokens, 12 heads, all of them: dQ 317 us without this, 427
// with every tile's product).
template <typename T, bool BIAS, int ST, int W, bool FEW>
__device__ __forceinline__ void ex_dq_block(const ExactParams& p, char* smem, int vt, int hx, int b, int Gp) {
  constexpr int ES = ExFmt<T>::ES, TB = tile_bytes<T>();
  const int n = 2 * p.D + 129;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* tb = reinterpret_cast<float*>(smem + kDqLds<T, ST, W>);  // [Gp][n]
  const int c = lane & 31, hf = lane >> 5;
  const ExRow0 br = ex_batch_row(p, b);
  const int hk = hx * Gp / p.G;

  const int v = vt * 32 + c, i = v / Gp, g = v % Gp, head = hx * Gp + g;
  const bool live = i < br.qlen;
  const int imin = vt * 32 / Gp, imax = min((vt * 32 + 31) / Gp, br.qlen - 1);
  const int pmin = br.pos + imin, pmax = br.pos + imax, pend = br.pos + (vt * 32 + 31) / Gp;
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
  for (int k = 0; k < ST - 1; ++k) load(wave + k * W, k);

  const int64_t hcol = head * kDHead;
  const char* qrow = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + hcol) * ES;
  const char* dyrow = static_cast<const char*>(p.dY.data) + (b * p.dY.batch + i * p.dY.row + hcol) * ES;
  const ExRow<T> q = live ? ex_global_row<T>(qrow, hf) : ex_zero_row<T>();
  const ExRow<T> dy = live ? ex_global_row<T>(dyrow, hf) : ex_zero_row<T>();
  float D = 0.f, cr = INFINITY;  // a row without keys, or behind the last query: every P is 0
  if (live) {
    const int64_t row = ((int64_t)b * p.H + head) * p.nq + i;
    if constexpr (ES == 2) {
      const char* yrow = static_cast<const char*>(p.Y.data) + (b * p.Y.batch + i * p.Y.row + hcol) * ES;
      D = ex_row_dot<T>(dy, ex_global_row<T>(yrow, hf), D);
      const float lse = p.lse[row];
      cr = ex_row_offset(lse);
    } else {  // k_exact_stats has been here
      cr = p.rowstat[row];
      D = p.rowstat[(int64_t)p.B * p.H * p.nq + row];
    }
  }
  if constexpr (ES == 2) D += ex_other_half(D);
  const int pos = br.pos + i;
  const ExSpan keys = ex_keys_of(p, pos, br.klen);
  const float* tl = nullptr;
  float rest = 0.f;  // sum of dS
  if constexpr (BIAS) {
    ex_fill_bias<T>(p, tb, hx * Gp, Gp);
    __syncthreads();
    tl = tb + g * n + p.D + 64;
  }
  f32x16_t dq[2] = {ex_zero16(), ex_zero16()}, pk[2] = {ex_zero16(), ex_zero16()};

  int slot = 0;
  for (int idx = wave; idx < tiles.n; idx += W) {
    wait_lds();  // the tile read last is overwritten by the next loads
    load(idx + (ST - 1) * W, slot == 0 ? ST - 1 : slot - 1);
    wait_vmcnt<(ST - 1) * 2 * ExFmt<T>::NL>();
    asm volatile("" ::: "memory");
    char* kt = smem + (wave * ST + slot) * 2 * TB;
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
      ex_mask(x, keys, k0 + 4 * hf, k0 > 0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = ex_exp2(x[r]);
    if constexpr (ES == 2) ex_cols_product<T>(pk, kt, x, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] *= dp[r] - D;
    ex_cols_product<T, FEW>(dq, kt, x, lane);
    if constexpr (ES == 2) rest += ex_sum16(x);
    slot = slot == ST - 1 ? 0 : slot + 1;
  }
  wait_vmcnt<0>();  // no load is under way into what is written next
  __syncthreads();
  float* ys = reinterpret_cast<float*>(smem);
  if constexpr (ES == 2) {
    float* rests = ys + W * 32 * kYS;  // [wave][row]
    rest += ex_other_half(rest);
    if (hf == 0) rests[wave * 32 + c] = rest;
    __syncthreads();
    rest = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) rest += rests[k * 32 + c];
    D += rest;
#pragma unroll
    for (int cc = 0; cc < 2; ++cc)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[cc][r] = fmaf(-rest, pk[cc][r], dq[cc][r]);
  }
  if (!ex_has(ex_many_keys(p, br.klen), pos)) dq[0] = dq[1] = ex_zero16();
  ex_put_sums(ys, dq, wave * 32 + c, hf);
  if constexpr (ES == 2)
    if (wave == 0 && hf == 0 && i < p.nq) ex_put_stat(p, ((int64_t)b * p.H + head) * p.nq + i, cr, D);
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 8 / W; ++half) {
    const int row = (threadIdx.x >> 4) + half * 4 * W, col = (threadIdx.x & 15) * 4;
    const int vr = vt * 32 + row, ir = vr / Gp;
    if (ir < p.nq)
      ex_store4(static_cast<T*>(p.dQ.data) + b * p.dQ.batch + ir * p.dQ.row + (hx * Gp + vr % Gp) * kDHead + col,
                ex_join_sums<W>(ys, row, col, p.scale));
  }
}

template <bool BIAS, int W, bool FEW>
__global__ __launch_bounds__(64 * W) void k_exact_dq(ExactParams p) {  // bf16
  extern __shared__ __align__(16) char smem[];
  const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp, bid = blockIdx.x / nvt;
  ex_dq_block<uint16_t, BIAS, 2, W, FEW>(p, smem, blockIdx.x % nvt, bid % Hx, bid / Hx, p.Gp);
}

// ------------------------------------------------------------------ dK, dV
// Blocks of 32 keys of a key head; the waves share the query tiles of all its query heads, or of the
// block's part of them (kv_splits). S = Q K^T and dP = dY V^T with the lane holding a key: P and dS
// feed dV^T = dY^T P and dK^T = Q^T dS. A wave loads its tiles of Q, dY and row statistics straight
// into LDS.
template <typename T, bool BIAS, int ST, int W, bool FEW>
__device__ __forceinline__ void ex_dkv_block(const ExactParams& p, char* smem, int kt, int hk, int b, int split, int splits,
                                             int64_t part, int heads_at_once) {
  constexpr int ES = ExFmt<T>::ES, TB = tile_bytes<T>(), SB = kDkvStage<T>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5, n = 2 * p.D + 129;
  ExDiag diag{reinterpret_cast<float*>(smem + kDkvLds<T, ST, W>) + wave * n, 0.f, -1};
  float* tb = reinterpret_cast<float*>(smem + kDkvLds<T, ST, W>) + W * n;  // [heads_at_once][n]
  const ExRow0 br = ex_batch_row(p, b);
  const int j = kt * 32 + c, jmax = min(kt * 32 + 31, br.klen - 1);
  const ExTiles tiles = ex_query_tiles(p, br, kt * 32, jmax);
  const ExSpan queries = ex_queries_of(p, br, j);
  const ExRange many = ex_many_keys(p, br.klen);

  const bool live = j < br.klen;
  const char* krow = static_cast<const char*>(p.K.data) + (b * p.K.batch + j * p.K.row + hk * kDHead) * ES;
  const char* vrow = static_cast<const char*>(p.V.data) + (b * p.V.batch + j * p.V.row + hk * kDHead) * ES;
  const ExRow<T> kf = live ? ex_global_row<T>(krow, hf) : ex_zero_row<T>();
  const ExRow<T> vf = live ? ex_global_row<T>(vrow, hf) : ex_zero_row<T>();
  f32x16_t dk[2] = {ex_zero16(), ex_zero16()}, dv[2] = {ex_zero16(), ex_zero16()};
  const uint32_t lds = lds_addr(smem) + (uint32_t)wave * ST * SB;
  const int all = tiles.n * p.G, from = ex_part(all, split, splits), to_ = ex_part(all, split + 1, splits);
  float far_l = 0.f, far_r = 0.f;
  part += wave;
  if constexpr (BIAS)
    for (int e = lane; e < n; e += 64) diag.dg[e] = 0.f;

  for (int g0 = 0; g0 < p.G; g0 += heads_at_once) {
    const int ng = min(heads_at_once, p.G - g0), h0 = hk * p.G + g0;
    if constexpr (BIAS) {
      __syncthreads();
      ex_fill_bias<T>(p, tb, h0, ng);
      __syncthreads();
    }
    const int total = min(to_ - g0 * tiles.n, tiles.n * ng), first = max(from - g0 * tiles.n, 0) + wave;
    int head = 0;  // of the chunk: whose sums along diagonals are under way
    auto load = [&](int idx, int slot) __attribute__((always_inline)) {  // past the last tile: zeros
      const int h = h0 + (tiles.n > 0 ? idx / tiles.n : 0);
      const int i0 = (tiles.n > 0 ? ex_tile_at(tiles, idx % tiles.n) : 0) * 32, limit = idx < total ? br.qlen : 0;
      const char* Qb = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + h * kDHead) * ES;
      const char* Yb = static_cast<const char*>(p.dY.data) + (b * p.dY.batch + h * kDHead) * ES;
      const uint32_t to = lds + slot * SB;
      ex_load_tile<T>(ex_rsrc(Qb, p.Q.row * ES, i0, limit, ExFmt<T>::RB), (int)p.Q.row * ES, to, lane);
      ex_load_tile<T>(ex_rsrc(Yb, p.dY.row * ES, i0, limit, ExFmt<T>::RB), (int)p.dY.row * ES, to + TB, lane);
      const char* st = reinterpret_cast<const char*>(p.rowstat + ((int64_t)b * p.H + h) * p.nq);
      ex_load_lds4(ex_rsrc(st, 4, i0, limit, 4), lane * 4, to + 2 * TB);
      ex_load_lds4(ex_rsrc(st + 4 * (int64_t)p.B * p.H * p.nq, 4, i0, limit, 4), lane * 4, to + 2 * TB + 256);
    };
#pragma unroll
    for (int k = 0; k < ST - 1; ++k) load(first + k * W, k);
    int slot = 0;
    for (int idx = first; idx < total; idx += W) {
      wait_lds();  // the tile read last is overwritten by the next loads
      load(idx + (ST - 1) * W, slot == 0 ? ST - 1 : slot - 1);
      wait_vmcnt<(ST - 1) * (2 * ExFmt<T>::NL + 2)>();
      asm volatile("" ::: "memory");
      const char* qt = smem + (wave * ST + slot) * SB;
      const float* stat = reinterpret_cast<const float*>(qt + 2 * TB);
      const int i0 = ex_tile_at(tiles, idx % tiles.n) * 32, p0 = br.pos + i0;
      f32x16_t x = ex_rows_product<T>(qt, kf, c, hf);
      f32x16_t ds = ex_rows_product<T>(qt + TB, vf, c, hf);
      float cr[16], D[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // rows 8 k + 4 hf ..
        const float4 t = *reinterpret_cast<const float4*>(stat + 8 * k + 4 * hf);
        const float4 u = *reinterpret_cast<const float4*>(stat + 64 + 8 * k + 4 * hf);
        cr[4 * k] = t.x, cr[4 * k + 1] = t.y, cr[4 * k + 2] = t.z, cr[4 * k + 3] = t.w;
        D[4 * k] = u.x, D[4 * k + 1] = u.y, D[4 * k + 2] = u.z, D[4 * k + 3] = u.w;
      }
      if constexpr (ES == 2) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          x[r] += cr[r];
          ds[r] += D[r];
          cr[r] = 0.f;
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] -= D[r];
      }
      ex_drop_single(ds, many, p0, hf);
      int side = 0;
      if constexpr (BIAS) {
        for (const int h = idx / tiles.n; head < h; ++head) {
          ex_put_buckets(p, diag, n, far_l, far_r, part, h0 + head, lane);
          far_l = far_r = 0.f;
        }
        const float* tl = tb + head * n + p.D + 64;
        side = ex_bias_side(p, kt * 32, p0, p0 + 31);
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
      // (without a bias gradient keys past the last one may have any P and dS, which are not stored)
      if (i0 + 32 > br.qlen || !ex_whole(p, p0, p0 + 31, kt * 32, BIAS ? br.klen : 0x7fffffff)) {
        ex_mask(x, queries, i0 + 4 * hf, p0 > 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = ex_exp2(x[r]);
        ds[r] *= x[r];
      }
      ex_cols_product<T, FEW>(dv, qt + TB, x, lane);
      ex_cols_product<T, FEW>(dk, qt, ds, lane);
      if constexpr (BIAS) {
        if (side < 0) far_l += ex_sum16(ds);
        else if (side > 0) far_r += ex_sum16(ds);
        else ex_diagonals(diag, ds, p.D + 64 + kt * 32 - p0, lane);
      }
      slot = slot == ST - 1 ? 0 : slot + 1;
    }
    if constexpr (BIAS)
      for (; head < ng; ++head) {
        ex_put_buckets(p, diag, n, far_l, far_r, part, h0 + head, lane);
        far_l = far_r = 0.f;
      }
    wait_vmcnt<0>();
  }
  __syncthreads();
  float* ys = reinterpret_cast<float*>(smem);  // one of the two at a time
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (which) __syncthreads();
    ex_put_sums(ys, which ? dv : dk, wave * 32 + c, hf);
    __syncthreads();
#pragma unroll
    for (int half = 0; half < 8 / W; ++half) {
      const int row = (threadIdx.x >> 4) + half * 4 * W, col = (threadIdx.x & 15) * 4, jr = kt * 32 + row;
      if (jr >= p.nk) continue;
      if (splits > 1) {
        const int64_t at = (((int64_t)(split * p.B + b) * p.nk + jr) * p.Hk + hk) * kDHead + col;
        ex_store4((which ? p.part_dv : p.part_dk) + at, ex_join_sums<W>(ys, row, col, 1.f));
      } else {
        const ExactOut& t = which ? p.dV : p.dK;
        const float4 v = ex_join_sums<W>(ys, row, col, which ? 1.f : p.scale);
        ex_store4(static_cast<T*>(t.data) + b * t.batch + jr * t.row + hk * kDHead + col,
                  jr < br.klen ? v : make_float4(0.f, 0.f, 0.f, 0.f));
      }
    }
  }
}

template <bool BIAS, int W, bool FEW>
__global__ __launch_bounds__(64 * W) void k_exact_dkv(ExactParams p, int heads_at_once) {  // bf16
  extern __shared__ __align__(16) char smem[];
  const int nkt = (p.nk + 31) / 32;
  int bid = blockIdx.x;
  const int kt = bid % nkt;
  bid /= nkt;
  const int hk = bid % p.Hk;
  bid /= p.Hk;
  const int64_t part = ((int64_t)bid * nkt + kt) * W;  // bid: split * B + batch row
  ex_dkv_block<uint16_t, BIAS, 2, W, FEW>(p, smem, kt, hk, bid % p.B, bid / p.B, p.kv_splits, part, heads_at_once);
}

// float32: both in one launch, behind k_exact_stats, the keys' blocks first.
template <bool BIAS>
__global__ __launch_bounds__(kExThreads) void k_exact_backward_f32(ExactParams p, int heads_at_once) {
  extern __shared__ __align__(16) char smem[];
  const int nkt = (p.nk + 31) / 32, keys = nkt * p.Hk * p.B * p.kv_splits;
  int bid = blockIdx.x;
  if (bid < keys) {
    const int kt = bid % nkt;
    bid /= nkt;
    const int hk = bid % p.Hk;
    bid /= p.Hk;
    const int64_t part = ((int64_t)bid * nkt + kt) * kExWaves;  // bid: split * B + batch row
    ex_dkv_block<float, BIAS, 1, kExWaves, false>(p, smem, kt, hk, bid % p.B, bid / p.B, p.kv_splits, part, heads_at_once);
  } else {
    bid -= keys;
    const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp, at = bid / nvt;
    ex_dq_block<float, BIAS, 1, kExWaves, false>(p, smem, bid % nvt, at % Hx, at / Hx, p.Gp);
  }
}

// ------------------------------------------------------------------ tiles of 64 rows, bf16
// For grids that fill the card: blocks of 128 rows, four waves of 32, that share the tiles they loop
// over, loaded straight into LDS two tiles ahead of their use (three buffers). Both kernels are
// software pipelined by half tiles of 32: a step has the matrix products of S and dP of half tile
// h + 1 in eight slots, each one MFMA beside the vector work of two pairs of h (P and dS), then the
// products that P and dS of h feed. The source fixes the order; an operand is read from LDS
// kAhead slots before its MFMA.
constexpr int kAhead = 4;

// One MFMA slot's vector work: pairs 2 j, 2 j + 1 of a half tile. The exp2 results of one slot are used
// in the next.
struct ExPair {
  float e0, e1;
};
template <bool FMA>  // FMA: a logit is fac * s + add, else fac * s
__device__ __forceinline__ ExPair ex_pair(const f32x16_t& s, int j, float fac, float add) {
  ExPair r;
  const float x0 = FMA ? __fmaf_rn(s[2 * j], fac, add) : s[2 * j] * fac;
  const float x1 = FMA ? __fmaf_rn(s[2 * j + 1], fac, add) : s[2 * j + 1] * fac;
  r.e0 = ex_exp2(x0);
  r.e1 = ex_exp2(x1);
  ex_pin(r.e0);
  ex_pin(r.e1);
  return r;
}

constexpr float kSmallP = 0x1p-6f;

template <bool BIAS, bool WIN, bool FEW>
__global__ __launch_bounds__(kExThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_exact_dq_tiles(ExactParams p) {
  extern __shared__ __align__(16) char smem[];  // three K tiles, three V tiles, the bias table
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5;
  float* tb = reinterpret_cast<float*>(smem + 6 * kTile64);
  int qt, pair;
  const int nqt = (p.nq + 127) / 128;
  int bid = blockIdx.x;
  if constexpr (WIN) {  // the first blocks: the rows around a global query
    if (bid < p.H * p.B) {
      const int first = ex_global_rows(p, ex_batch_row(p, bid / p.H));
      if (first >= 0) ex_dq_block<uint16_t, BIAS, 2, 4, false>(p, smem, first / 32, bid % p.H, bid / p.H, 1);
      return;
    }
    bid -= p.H * p.B;
  }
  ex_block_pair(bid, nqt, p.H * p.B, p.causal || p.window, qt, pair);
  if (p.causal) qt = nqt - 1 - qt;  // the longest rows first
  const int h = pair % p.H, b = pair / p.H, hk = h / p.G;
  const ExRow0 br = ex_batch_row(p, b);
  const int qw = qt * 128 + wave * 32, i = qw + c;
  const int global = WIN ? ex_global_rows(p, br) : -1;
  const int first = qt * 128 + (WIN && global == qt * 128 ? 32 : 0), last = min(qt * 128 + 128, br.qlen) - 1;
  const ExTiles tiles = last >= first ? ex_key_tiles<64>(p, br.pos + first, br.pos + last, br.klen, !WIN) : ExTiles{-1, 0, 0};
  const ExRange whole = ex_whole_keys(p, br.pos + qw, br.pos + min(qw + 32, br.qlen) - 1, br.klen);

  const char* Kb = static_cast<const char*>(p.K.data) + (b * p.K.batch + hk * kDHead) * 2;
  const char* Vb = static_cast<const char*>(p.V.data) + (b * p.V.batch + hk * kDHead) * 2;
  const int kpitch = (int)p.K.row * 2, vpitch = (int)p.V.row * 2;
  const uint32_t kl = ex_load64(wave, lane, kpitch), vl = ex_load64(wave, lane, vpitch), lds = lds_addr(smem);
  // Tile t into buffer `slot`, in the order of t; past the last tile: zeros
  ExStream ks, vs;
  auto load = [&](int t, int slot) __attribute__((always_inline)) {
    if (t == 0 || (tiles.first >= 0 && t == 1)) {
      ks = ex_stream(Kb, kpitch, ex_tile_at(tiles, t) * 64, br.klen);
      vs = ex_stream(Vb, vpitch, ex_tile_at(tiles, t) * 64, br.klen);
    }
    if (t >= tiles.n) ks.rows = vs.rows = 0;
    ex_load_next64(ks, kpitch, kl, lds + slot * kTile64, wave);
    ex_load_next64(vs, vpitch, vl, lds + (3 + slot) * kTile64, wave);
  };
  load(0, 0);
  const bool live = i < br.qlen;
  const int64_t hcol = h * kDHead;
  ExRow<uint16_t> q = ex_zero_row<uint16_t>(), dy = q;
  float D = 0.f, cr = INFINITY;  // a row without keys, or behind the last query: every P is 0
  if (live) {
    q = ex_global_row<uint16_t>(static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + hcol) * 2, hf);
    dy = ex_global_row<uint16_t>(static_cast<const char*>(p.dY.data) + (b * p.dY.batch + i * p.dY.row + hcol) * 2, hf);
    D = ex_row_dot<uint16_t>(
        dy, ex_global_row<uint16_t>(static_cast<const char*>(p.Y.data) + (b * p.Y.batch + i * p.Y.row + hcol) * 2, hf), D);
    const float lse = p.lse[((int64_t)b * p.H + h) * p.nq + i];
    cr = ex_row_offset(lse);
  }
  load(1, 1);
  D += ex_other_half(D);
  f32x16_t nD;  // where dP's sums start (FEW: at 0, and D is taken off afterwards, which leaves registers for dS)
#pragma unroll
  for (int r = 0; r < 16; ++r) nD[r] = FEW ? 0.f : -D;
  const float* tl = tb + p.D + 64;
  float rest = 0.f;  // sum of dS
  if constexpr (BIAS) {
    ex_fill_bias<uint16_t>(p, tb, h, 1);
    __syncthreads();
  }

  const ExRows64 ra = ex_rows64(lane);
  const ExCols64<false> ca = ex_cols64<false>(lane);
  const f32x16_t zero = ex_zero16();
  f32x16_t dq[2] = {zero, zero}, pk[2] = {zero, zero}, s0, s1, p0, p1;
  u32x4_t fr[kAhead], ds[2];
  f32x16_t pr;
  // Operand of slot j: K, V chunk j / 2 in turn of half tile (kt, half), then K columns of (ct, chalf).
  auto read = [&](int j, const char* kt, int half, const char* ct, int chalf) __attribute__((always_inline)) {
    if (j < 8) return ex_read_row(kt + (j & 1) * 3 * kTile64, ra, half, j >> 1);
    return ex_read_col(ct, ca, chalf, (j - 8) >> 1, j & 1);
  };
  float fac = p.s2, add = -cr;
  // What a half tile's scores still need: masks and the bias of near pairs.
  auto fix = [&](f32x16_t& s, int k0) __attribute__((always_inline)) {
    if constexpr (BIAS) {
      const int side = ex_bias_side(p, k0, br.pos + qw, br.pos + qw + 31);
      if (side != 0) {
        fac = p.s2;
        add = tl[side * p.D] - cr;
      } else {
        fac = 1.f;
        add = -cr;
        const float* at = tl + (k0 + 4 * hf - br.pos - qw - ex_opaque(c));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __fmaf_rn(s[r], p.s2, at[(r & 3) + 8 * (r >> 2)]);
      }
    }
    if (__builtin_expect(!ex_has(whole, k0), 0)) {
      const ExSpan keys = ex_keys_of(p, br.pos + qw + ex_opaque(c), br.klen);
      ex_mask(s, keys, k0 + 4 * hf, k0 > 0);
    }
  };
  // Half tile `ch` of ct: dS from (s, d); half tile nh of nt: S and dP into (sn, dn). (ft, fh): the one after that.
  auto step = [&](f32x16_t& s, f32x16_t& d, f32x16_t& sn, f32x16_t& dn, const char* ct, int ch, const char* nt, int nh,
                  const char* ft, int fh) __attribute__((always_inline)) {
    ExPair e{0.f, 0.f};
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < 12; ++j) {
      if (j < 8) {
        if (j % 2 == 0) sn = ex_mfma<uint16_t>(fr[j % kAhead], q.v[j >> 1], j == 0 ? zero : sn);
        else dn = ex_mfma<uint16_t>(fr[j % kAhead], dy.v[j >> 1], j == 1 ? nD : dn);
      } else {
        dq[j & 1] = ex_mfma<uint16_t>(fr[j % kAhead], ds[(j - 8) >> 1], dq[j & 1]);
      }
      __builtin_amdgcn_sched_barrier(0);  // the read takes the registers the MFMA has read
      fr[j % kAhead] = j + kAhead < 12 ? read(j + kAhead, nt, nh, ct, ch) : read(j + kAhead - 12, ft, fh, nullptr, 0);
      if (j <= 8) {
        const ExPair b4 = e;
        if (j < 8) e = ex_pair<true>(s, j, fac, add);
        if (j > 0) {
          const int k = j - 1;
          d[2 * k] = (FEW ? d[2 * k] - D : d[2 * k]) * b4.e0;
          d[2 * k + 1] = (FEW ? d[2 * k + 1] - D : d[2 * k + 1]) * b4.e1;
          rest += d[2 * k] + d[2 * k + 1];
          pr[2 * k] = b4.e0;
          pr[2 * k + 1] = b4.e1;
          most = fmaxf(fmaxf(most, b4.e0), b4.e1);
          uint32_t w = pack_bf16x2(d[2 * k], d[2 * k + 1]);
          ex_pin(w);
          ds[k >> 2][k & 3] = w;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (FEW) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u32x4_t w;
#pragma unroll
        for (int l = 0; l < 4; ++l) w[l] = ex_pack_rest(d[8 * k + 2 * l], d[8 * k + 2 * l + 1], ds[k][l]);
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) dq[cc] = ex_mfma<uint16_t>(ex_read_col(ct, ca, ch, k, cc), w, dq[cc]);
      }
    }
    if (__builtin_expect(__any(most > kSmallP), 0)) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u32x4_t w;
#pragma unroll
        for (int l = 0; l < 4; ++l) w[l] = pack_bf16x2(pr[8 * k + 2 * l], pr[8 * k + 2 * l + 1]);
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) pk[cc] = ex_mfma<uint16_t>(ex_read_col(ct, ca, ch, k, cc), w, pk[cc]);
      }
    }
  };

  wait_vmcnt<4>();  // tile 0
  stage_barrier();
  s0 = zero;
  p0 = nD;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const u32x4_t f = read(j, smem, 0, nullptr, 0);
    if (j % 2 == 0) s0 = ex_mfma<uint16_t>(f, q.v[j >> 1], s0);
    else p0 = ex_mfma<uint16_t>(f, dy.v[j >> 1], p0);
  }
#pragma unroll
  for (int j = 0; j < kAhead; ++j) fr[j] = read(j, smem, 1, nullptr, 0);
  int b0 = 0, b1 = 1, b2 = 2;  // buffers of tiles t, t + 1, t + 2
#pragma clang loop unroll(disable)
  for (int t = 0; t < tiles.n; ++t) {
    wait_vmcnt<0>();
    stage_barrier();
    load(t + 2, b2);
    const char *ct = smem + b0 * kTile64, *nt = smem + b1 * kTile64;
    const int k0 = ex_tile_at(tiles, t) * 64;
    fix(s0, k0);
    step(s0, p0, s1, p1, ct, 0, ct, 1, nt, 0);
    fix(s1, k0 + 32);
    step(s1, p1, s0, p0, ct, 1, nt, 0, nt, 1);
    const int o = b0;
    b0 = b1;
    b1 = b2;
    b2 = o;
  }
  rest += ex_other_half(rest);
  D += rest;
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[cc][r] = fmaf(-rest, pk[cc][r], dq[cc][r]);
  if (!ex_has(ex_many_keys(p, br.klen), br.pos + i)) dq[0] = dq[1] = zero;
  wait_vmcnt<0>();  // no load is under way into what is written next
  __syncthreads();
  if (WIN && qw == global) return;  // another block has these rows
  if (hf == 0 && i < p.nq) ex_put_stat(p, ((int64_t)b * p.H + h) * p.nq + i, cr, D);
  char* out = static_cast<char*>(p.dQ.data) + (b * p.dQ.batch + (int64_t)qw * p.dQ.row + hcol) * 2;
  ex_store_rows32(smem + wave * 32 * 144, dq, p.scale, out, p.dQ.row * 2, p.nq - qw, lane);
}

constexpr int kDkvTilesStage = 2 * kTile64 + 512;  // Q, dY, two planes of 64 statistics
constexpr int kDkvTilesLds = 3 * kDkvTilesStage;

template <bool BIAS, bool WIN, bool FEW>
__global__ __launch_bounds__(kExThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_exact_dkv_tiles(ExactParams p, int heads_at_once) {
  extern __shared__ __align__(16) char smem[];  // three stages, sums along diagonals, the bias tables of `heads_at_once` heads
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5, n = 2 * p.D + 129;
  const int nkt = (p.nk + 127) / 128;
  ExDiag diag{reinterpret_cast<float*>(smem + kDkvTilesLds) + wave * n, 0.f, -1};
  float* tb = reinterpret_cast<float*>(smem + kDkvTilesLds) + kExWaves * n;
  int kt, pair;
  int bid = blockIdx.x;
  if constexpr (WIN) {  // the first blocks: the keys around the global one (kv_splits is 1)
    if (bid < p.Hk * p.B) {
      const int64_t part = ((int64_t)p.B * nkt + bid / p.Hk) * kExWaves;
      ex_dkv_block<uint16_t, BIAS, 2, 4, false>(p, smem, 0, bid % p.Hk, bid / p.Hk, 0, 1, part, heads_at_once);
      return;
    }
    bid -= p.Hk * p.B;
  }
  ex_block_pair(bid, nkt, p.Hk * p.B * p.kv_splits, p.causal || p.window, kt, pair);
  const int hk = pair % p.Hk, b = pair / p.Hk % p.B, split = pair / (p.Hk * p.B);
  const ExRow0 br = ex_batch_row(p, b);
  const int kw = kt * 128 + wave * 32, j = kw + c;
  const ExTiles tiles = ex_query_tiles<64>(p, br, kt * 128 + (WIN && kt == 0 ? 32 : 0), min(kt * 128 + 128, br.klen) - 1);

  ExRow<uint16_t> kf = ex_zero_row<uint16_t>(), vf = kf;
  if (j < br.klen) {
    kf = ex_global_row<uint16_t>(static_cast<const char*>(p.K.data) + (b * p.K.batch + j * p.K.row + hk * kDHead) * 2, hf);
    vf = ex_global_row<uint16_t>(static_cast<const char*>(p.V.data) + (b * p.V.batch + j * p.V.row + hk * kDHead) * 2, hf);
  }
  const int qpitch = (int)p.Q.row * 2, ypitch = (int)p.dY.row * 2;
  const uint32_t ql = ex_load64(wave, lane, qpitch), yl = ex_load64(wave, lane, ypitch), lds = lds_addr(smem);
  const ExRows64 ra = ex_rows64(lane);
  const ExCols64<false> ca = ex_cols64<false>(lane);
  const f32x16_t zero = ex_zero16();
  f32x16_t dk[2] = {zero, zero}, dv[2] = {zero, zero}, s0, s1, p0, p1;
  u32x4_t fr[kAhead], pp[2], ds[2];
  // Operand of slot i: Q, dY chunk i / 2 in turn of half tile (rt, half); then, for each 16 rows of
  // (ct, chalf), dY's two column halves and Q's.
  auto read = [&](int i, const char* rt, int half, const char* ct, int chalf) __attribute__((always_inline)) {
    if (i < 8) return ex_read_row(rt + (i & 1) * kTile64, ra, half, i >> 1);
    return ex_read_col(ct + ((i & 2) ? 0 : kTile64), ca, chalf, (i - 8) >> 2, i & 1);
  };
  // Rows of a half tile: where S and dP start, -c / s2 and -D.
  auto start = [&](f32x16_t& s, f32x16_t& d, const char* rt, int half) __attribute__((always_inline)) {
    const float* at = reinterpret_cast<const float*>(rt + 2 * kTile64) + 32 * half + 4 * hf;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 t = *reinterpret_cast<const float4*>(at + 8 * k), u = *reinterpret_cast<const float4*>(at + 64 + 8 * k);
      s[4 * k] = t.x, s[4 * k + 1] = t.y, s[4 * k + 2] = t.z, s[4 * k + 3] = t.w;
      d[4 * k] = u.x, d[4 * k + 1] = u.y, d[4 * k + 2] = u.z, d[4 * k + 3] = u.w;
    }
  };
  const bool mine = !WIN || kw > 0;  // another block has the first 32 keys
  ExRange whole = ex_whole_queries(p, kw, !mine ? 0 : BIAS ? br.klen : 0x7fffffff);
  // rows past the last query come as zeros, scores and offsets too: under a bias their P is what exp makes of the
  // bias alone, which may pass float32's range (without one it is 1, times zeros)
  if constexpr (BIAS) whole.hi = min(whole.hi, br.pos + br.qlen - 32);
  const ExRange many = ex_many_keys(p, br.klen);
  float fac = p.s2, add = 0.f, far_l = 0.f, far_r = 0.f;
  int side = 0, entry = 0;  // where the half tile lies, and the entry of its first key and query
  const float* tl = nullptr;
  const int64_t part = ((int64_t)(split * p.B + b) * nkt + kt) * kExWaves + wave;
  if constexpr (BIAS)
    for (int e = lane; e < n; e += 64) diag.dg[e] = 0.f;
  // The bias of the half tile whose scores come next, read before they are there: near pairs' entries.
  int next = 0;
  f32x16_t bv;
  auto peek = [&](int i0, const float* tn) __attribute__((always_inline)) {
    const int q0 = br.pos + i0;
    next = ex_bias_side(p, kw, q0, q0 + 31);
    if (next == 0) {
      const float* at = tn + (kw + ex_opaque(c) - q0 - 4 * hf);
#pragma unroll
      for (int r = 0; r < 16; ++r) bv[r] = at[-((r & 3) + 8 * (r >> 2))];
    }
  };
  auto fix = [&](f32x16_t& s, f32x16_t& d, int i0) __attribute__((always_inline)) {
    const int q0 = br.pos + i0;
    ex_drop_single(d, many, q0, hf);
    if constexpr (BIAS) {
      side = next;
      entry = p.D + 64 + kw - q0;
      fac = p.s2;
      add = 0.f;
      if (side != 0) {
        add = tl[side * p.D];
      } else {
        fac = 1.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __fmaf_rn(s[r], p.s2, bv[r]);
      }
    }
    // without a bias rows past the last query add nothing, and keys past the last key nothing that is stored
    if (__builtin_expect(!ex_has(whole, q0), 0)) {
      const ExSpan queries = mine ? ex_queries_of(p, br, kw + ex_opaque(c)) : ex_span(0, -1, -1);
      ex_mask(s, queries, i0 + 4 * hf, q0 > 0);
    }
  };
  // Half tile ch of ct: P and dS from (s, d); half tile nh of nt, of queries in on and bias table tn: S and dP into
  // (sn, dn); (ft, fh): the one after that, whose start values take the place of (s, d).
  auto step = [&](f32x16_t& s, f32x16_t& d, f32x16_t& sn, f32x16_t& dn, const char* ct, int ch, const char* nt, int nh,
                  const char* ft, int fh, int in, const float* tn) __attribute__((always_inline)) {
    ExPair e{0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < 8) {
        if (i % 2 == 0) sn = ex_mfma<uint16_t>(fr[i % kAhead], kf.v[i >> 1], sn);
        else dn = ex_mfma<uint16_t>(fr[i % kAhead], vf.v[i >> 1], dn);
      } else if (i & 2) {
        dk[i & 1] = ex_mfma<uint16_t>(fr[i % kAhead], ds[(i - 8) >> 2], dk[i & 1]);
      } else {
        dv[i & 1] = ex_mfma<uint16_t>(fr[i % kAhead], pp[(i - 8) >> 2], dv[i & 1]);
      }
      __builtin_amdgcn_sched_barrier(0);  // the read takes the registers the MFMA has read
      fr[i % kAhead] = i + kAhead < 16 ? read(i + kAhead, nt, nh, ct, ch) : read(i + kAhead - 16, ft, fh, nullptr, 0);
      if (i <= 8) {
        const ExPair b4 = e;
        if (i < 8) e = ex_pair<BIAS>(s, i, fac, add);
        if (i > 0) {
          const int k = i - 1;
          d[2 * k] *= b4.e0;
          d[2 * k + 1] *= b4.e1;
          uint32_t w = pack_bf16x2(b4.e0, b4.e1), x = pack_bf16x2(d[2 * k], d[2 * k + 1]);
          ex_pin(w);
          ex_pin(x);
          pp[k >> 2][k & 3] = w;
          ds[k >> 2][k & 3] = x;
          if constexpr (FEW) s[2 * k] = b4.e0, s[2 * k + 1] = b4.e1;
        }
      }
      if (BIAS && i == 8) {
        if (side < 0) far_l += ex_sum16(d);
        else if (side > 0) far_r += ex_sum16(d);
        else ex_diagonals(diag, d, entry, lane);
      }
      if (!FEW && i == 9) start(s, d, ft, fh);
      if (BIAS && !FEW && i == 10) peek(in, tn);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (FEW) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        u32x4_t w, x;
#pragma unroll
        for (int l = 0; l < 4; ++l) {
          w[l] = ex_pack_rest(s[8 * k + 2 * l], s[8 * k + 2 * l + 1], pp[k][l]);
          x[l] = ex_pack_rest(d[8 * k + 2 * l], d[8 * k + 2 * l + 1], ds[k][l]);
        }
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) {
          dv[cc] = ex_mfma<uint16_t>(ex_read_col(ct + kTile64, ca, ch, k, cc), w, dv[cc]);
          dk[cc] = ex_mfma<uint16_t>(ex_read_col(ct, ca, ch, k, cc), x, dk[cc]);
        }
      }
      start(s, d, ft, fh);
      if constexpr (BIAS) peek(in, tn);
    }
  };

  const int all = tiles.n * p.G, from = ex_part(all, split, p.kv_splits), to_ = ex_part(all, split + 1, p.kv_splits);
  for (int g0 = 0; g0 < p.G; g0 += heads_at_once) {
    const int ng = min(heads_at_once, p.G - g0), h0 = hk * p.G + g0;
    const int first = max(from - g0 * tiles.n, 0), total = min(to_ - g0 * tiles.n, tiles.n * ng) - first;
    int g = 0, t = 0;  // head of the chunk and tile in use
    if (total > 0) {
    g = first / tiles.n;
    t = first % tiles.n;
    // the next tile to load (head lg, tile lt), and how many
    int lg = g, lt = t, left = total;
    bool jump = true;
    ExStream qs, ys;
    const char* stat = nullptr;  // of the wave's plane, for the tile
    auto load = [&](int slot) __attribute__((always_inline)) {  // past the last tile: zeros
      if (jump) {
        const int h = h0 + min(lg, ng - 1), i0 = ex_tile_at(tiles, lt) * 64;
        qs = ex_stream(static_cast<const char*>(p.Q.data) + (b * p.Q.batch + h * kDHead) * 2, qpitch, i0, br.qlen);
        ys = ex_stream(static_cast<const char*>(p.dY.data) + (b * p.dY.batch + h * kDHead) * 2, ypitch, i0, br.qlen);
        stat = reinterpret_cast<const char*>(p.rowstat + ((int64_t)(wave & 1) * p.B * p.H + (int64_t)b * p.H + h) * p.nq + i0);
      }
      if (left <= 0) qs.rows = ys.rows = 0;
      const uint32_t to = lds + slot * kDkvTilesStage;
      if (wave < 2) {  // a plane of statistics each
        const uint64_t a = (uint64_t)(uintptr_t)stat;
        u32x4_t rs;
        rs[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
        rs[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu));
        rs[2] = (uint32_t)__builtin_amdgcn_readfirstlane(max(min(qs.rows, 64), 0) * 4);
        rs[3] = 0x00020000u;
        ex_load_lds4(rs, lane * 4, to + 2 * kTile64 + 256 * wave);
      }
      ex_load_next64(qs, qpitch, ql, to, wave);
      ex_load_next64(ys, ypitch, yl, to + kTile64, wave);
      stat += 256;
      --left;
      ++lt;
      jump = lt == tiles.n || (tiles.first >= 0 && lt == 1);
      if (lt == tiles.n) {
        lt = 0;
        ++lg;
      }
    };
    __syncthreads();  // the buffers (and the bias tables) are this chunk's from here on
    load(0);
    load(1);
    if constexpr (BIAS) {
      ex_fill_bias<uint16_t>(p, tb, h0, ng);
      for (int k = 0; k < g; ++k) ex_put_buckets(p, diag, n, 0.f, 0.f, part, h0 + k, lane);
      tl = tb + g * n + p.D + 64;
      lds_barrier();
    }
    wait_vmcnt<4>();  // tile 0
    stage_barrier();
    start(s0, p0, smem, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32x4_t f = read(i, smem, 0, nullptr, 0);
      if (i % 2 == 0) s0 = ex_mfma<uint16_t>(f, kf.v[i >> 1], s0);
      else p0 = ex_mfma<uint16_t>(f, vf.v[i >> 1], p0);
    }
    start(s1, p1, smem, 1);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fr[i] = read(i, smem, 1, nullptr, 0);
    if constexpr (BIAS) peek(ex_tile_at(tiles, t) * 64, tl);
    int b0 = 0, b1 = 1, b2 = 2;  // buffers of the tile, the next one, the one after
#pragma clang loop unroll(disable)
    for (int it = 0; it < total; ++it) {
      wait_vmcnt<0>();
      stage_barrier();
      load(b2);
      const char *ct = smem + b0 * kDkvTilesStage, *nt = smem + b1 * kDkvTilesStage;
      const bool last = t + 1 == tiles.n;  // the next tile is the next head's first
      const int i0 = ex_tile_at(tiles, t) * 64, in = ex_tile_at(tiles, last ? 0 : t + 1) * 64;
      fix(s0, p0, i0);
      step(s0, p0, s1, p1, ct, 0, ct, 1, nt, 0, i0 + 32, tl);
      fix(s1, p1, i0 + 32);
      step(s1, p1, s0, p0, ct, 1, nt, 0, nt, 1, in, last && g + 1 < ng ? tl + n : tl);
      const int o = b0;
      b0 = b1;
      b1 = b2;
      b2 = o;
      if (++t == tiles.n) {
        t = 0;
        if constexpr (BIAS) {
          ex_put_buckets(p, diag, n, far_l, far_r, part, h0 + g, lane);
          far_l = far_r = 0.f;
          tl += n;
        }
        ++g;
      }
    }
    wait_vmcnt<0>();  // no load is under way into what is written next
    }
    if constexpr (BIAS)
      for (; g < ng; ++g) {  // what is left of the part's last head, and the heads behind it
        ex_put_buckets(p, diag, n, far_l, far_r, part, h0 + g, lane);
        far_l = far_r = 0.f;
      }
  }
  __syncthreads();
  if (!mine) return;
  if (p.kv_splits > 1) {
    if (j < p.nk) {
      const int64_t at = (((int64_t)(split * p.B + b) * p.nk + j) * p.Hk + hk) * kDHead + 4 * hf;
#pragma unroll
      for (int cc = 0; cc < 2; ++cc)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int64_t o = at + 32 * cc + 2 * r;
          *reinterpret_cast<float4*>(p.part_dk + o) = make_float4(dk[cc][r], dk[cc][r + 1], dk[cc][r + 2], dk[cc][r + 3]);
          *reinterpret_cast<float4*>(p.part_dv + o) = make_float4(dv[cc][r], dv[cc][r + 1], dv[cc][r + 2], dv[cc][r + 3]);
        }
    }
    return;
  }
  if (j >= br.klen) dk[0] = dk[1] = dv[0] = dv[1] = zero;
  char* st = smem + wave * 32 * 144;
  char* out = static_cast<char*>(p.dK.data) + (b * p.dK.batch + (int64_t)kw * p.dK.row + hk * kDHead) * 2;
  ex_store_rows32(st, dk, p.scale, out, p.dK.row * 2, p.nk - kw, lane);
  out = static_cast<char*>(p.dV.data) + (b * p.dV.batch + (int64_t)kw * p.dV.row + hk * kDHead) * 2;
  ex_store_rows32(st, dv, 1.f, out, p.dV.row * 2, p.nk - kw, lane);
}

// ------------------------------------------------------------------ up to 128 queries and keys, bf16
// One launch for all three gradients: a block has a (batch row, head)'s Q, K, V and dY in LDS, its four waves
// take 32 queries each for D and dQ, and then 32 keys each for dK and dV. What two launches cost at this size is
// mostly their starts and loads (backward pass, 12 heads, two launches against one: 1 x 32 tokens 13.1 and 7.4
// us; 1 x 128 13.3 and 10.4; 32 x 128 23.6 and 17.9; 128 x 128 69 and 48).
template <bool FEW>
__global__ __launch_bounds__(kExThreads) __attribute__((amdgpu_waves_per_eu(2))) void k_exact_backward_small(ExactParams p) {
  using T = uint16_t;
  extern __shared__ __align__(16) char smem[];  // Q, K, V, dY; -c / s2 and -D per query
  const int rows = exact_small_rows(p), M = rows * 128;
  char *Qs = smem, *Ks = smem + M, *Vs = smem + 2 * M, *Ys = smem + 3 * M;
  float* stat = reinterpret_cast<float*>(smem + 4 * M);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5, h = blockIdx.x % p.H, b = blockIdx.x / p.H, r0 = 32 * wave;
  const ExRow0 br = ex_batch_row(p, b);
  const int64_t hcol = h * kDHead;
  const uint32_t to = lds_addr(smem) + 4096u * wave;
  auto load = [&](const ExactRows& m, int limit, uint32_t at) __attribute__((always_inline)) {
    const char* base = static_cast<const char*>(m.data) + (b * m.batch + hcol) * 2;
    ex_load_tile<T>(ex_rsrc(base, m.row * 2, r0, limit, 128), (int)m.row * 2, to + at, lane);
  };
  load(p.K, br.klen, M);
  load(p.V, br.klen, 2 * M);
  load(p.Q, br.qlen, 0);
  load(p.dY, br.qlen, 3 * M);
  const int i = r0 + c;
  float D = 0.f, cr = INFINITY;  // a row without keys, or behind the last query: every P is 0
  if (i < br.qlen) {
    const char* y = static_cast<const char*>(p.Y.data) + (b * p.Y.batch + i * p.Y.row + hcol) * 2;
    const char* g = static_cast<const char*>(p.dY.data) + (b * p.dY.batch + i * p.dY.row + hcol) * 2;
    D = ex_row_dot<T>(ex_global_row<T>(g, hf), ex_global_row<T>(y, hf), D);
    const float lse = p.lse[((int64_t)b * p.H + h) * p.nq + i];
    cr = ex_row_offset(lse);
  }
  D += ex_other_half(D);
  wait_vmcnt<0>();
  __syncthreads();

  const int last = min(r0 + 32, br.qlen) - 1, pos = br.pos + i;
  const ExRange many = ex_many_keys(p, br.klen);
  f32x16_t dq[2] = {ex_zero16(), ex_zero16()};
  if (last >= r0) {  // wave-uniform
    const ExTiles tiles = ex_key_tiles(p, br.pos + r0, br.pos + last, br.klen);
    const ExSpan keys = ex_keys_of(p, pos, br.klen);
    ExRow<T> q, dy;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      q.v[g] = ex_tile_chunk<T>(Qs + 4096 * wave, c, hf, g);
      dy.v[g] = ex_tile_chunk<T>(Ys + 4096 * wave, c, hf, g);
    }
    f32x16_t pk[2] = {ex_zero16(), ex_zero16()};
    float rest = 0.f;
#pragma clang loop unroll(disable)
    for (int t = 0; t < tiles.n; ++t) {
      const int kt = ex_tile_at(tiles, t), k0 = 32 * kt;
      f32x16_t x = ex_rows_product<T>(Ks + 4096 * kt, q, c, hf);
      const f32x16_t dp = ex_rows_product<T>(Vs + 4096 * kt, dy, c, hf);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, -cr);
      if (!ex_whole(p, br.pos + r0, br.pos + last, k0, br.klen)) ex_mask(x, keys, k0 + 4 * hf, k0 > 0);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = ex_exp2(x[r]);
      ex_cols_product<T>(pk, Ks + 4096 * kt, x, lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= dp[r] - D;
      rest += ex_sum16(x);
      ex_cols_product<T, FEW>(dq, Ks + 4096 * kt, x, lane);
    }
    rest += ex_other_half(rest);  // the exact D less this one
    D += rest;
#pragma unroll
    for (int cc = 0; cc < 2; ++cc)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[cc][r] = fmaf(-rest, pk[cc][r], dq[cc][r]);
    if (!ex_has(many, pos)) dq[0] = dq[1] = ex_zero16();
  }
  if (hf == 0) {
    stat[i] = -cr * (1.f / p.s2);
    stat[rows + i] = -D;
  }
  __syncthreads();

  f32x16_t dk[2] = {ex_zero16(), ex_zero16()}, dv[2] = {ex_zero16(), ex_zero16()};
  const int jmax = min(r0 + 32, br.klen) - 1;
  if (jmax >= r0) {
    const ExTiles tiles = ex_query_tiles(p, br, r0, jmax);
    const ExSpan queries = ex_queries_of(p, br, r0 + c);
    ExRow<T> kf, vf;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      kf.v[g] = ex_tile_chunk<T>(Ks + 4096 * wave, c, hf, g);
      vf.v[g] = ex_tile_chunk<T>(Vs + 4096 * wave, c, hf, g);
    }
#pragma clang loop unroll(disable)
    for (int t = 0; t < tiles.n; ++t) {
      const int qt = ex_tile_at(tiles, t), i0 = 32 * qt, p0 = br.pos + i0;
      f32x16_t x = ex_rows_product<T>(Qs + 4096 * qt, kf, c, hf);
      f32x16_t ds = ex_rows_product<T>(Ys + 4096 * qt, vf, c, hf);
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // rows 8 k + 4 hf ..
        const float4 u = *reinterpret_cast<const float4*>(stat + i0 + 8 * k + 4 * hf);
        const float4 w = *reinterpret_cast<const float4*>(stat + rows + i0 + 8 * k + 4 * hf);
        x[4 * k] += u.x, x[4 * k + 1] += u.y, x[4 * k + 2] += u.z, x[4 * k + 3] += u.w;
        ds[4 * k] += w.x, ds[4 * k + 1] += w.y, ds[4 * k + 2] += w.z, ds[4 * k + 3] += w.w;
      }
      ex_drop_single(ds, many, p0, hf);
      if (i0 + 32 > br.qlen || !ex_whole(p, p0, p0 + 31, r0, 0x7fffffff)) ex_mask(x, queries, i0 + 4 * hf, p0 > 0);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[r] = ex_exp2(x[r] * p.s2);
        ds[r] *= x[r];
      }
      ex_cols_product<T, FEW>(dv, Ys + 4096 * qt, x, lane);
      ex_cols_product<T, FEW>(dk, Qs + 4096 * qt, ds, lane);
    }
  }
  __syncthreads();
  if (i >= br.klen) dk[0] = dk[1] = dv[0] = dv[1] = ex_zero16();
  char* st = smem + wave * 32 * 144;
  char* out = static_cast<char*>(p.dQ.data) + (b * p.dQ.batch + (int64_t)r0 * p.dQ.row + hcol) * 2;
  ex_store_rows32(st, dq, p.scale, out, p.dQ.row * 2, p.nq - r0, lane);
  out = static_cast<char*>(p.dK.data) + (b * p.dK.batch + (int64_t)r0 * p.dK.row + hcol) * 2;
  ex_store_rows32(st, dk, p.scale, out, p.dK.row * 2, p.nk - r0, lane);
  out = static_cast<char*>(p.dV.data) + (b * p.dV.batch + (int64_t)r0 * p.dV.row + hcol) * 2;
  ex_store_rows32(st, dv, 1.f, out, p.dV.row * 2, p.nk - r0, lane);
}

// Adds up what k_exact_dkv leaves in parts: the first `sums` blocks the bias gradient, one (bucket, head)
// per wave; the others dK and dV, four columns of a key per thread.
template <typename T>
__global__ __launch_bounds__(kExThreads) void k_exact_join_grads(ExactParams p, int sums) {
  const int lane = threadIdx.x & 63;
  if ((int)blockIdx.x < sums) {
    const int e = blockIdx.x * kExWaves + (threadIdx.x >> 6);  // bucket * H + head
    if (e >= p.buckets * p.H) return;
    float sum = 0.f;
    for (int k = lane; k < p.bias_parts; k += 64) sum += p.part_bias[(int64_t)k * p.buckets * p.H + e];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane != 0) return;
    if constexpr (ExFmt<T>::ES == 2) static_cast<T*>(p.dtable)[e] = (T)f32_to_bf16_bits(sum);
    else static_cast<T*>(p.dtable)[e] = sum;
    return;
  }
  const int64_t all = (int64_t)p.B * p.nk * p.Hk * kDHead, e = ((int64_t)(blockIdx.x - sums) * kExThreads + threadIdx.x) * 4;
  if (e >= all) return;
  const int col = (int)(e % (p.Hk * kDHead));
  const int64_t row = e / (p.Hk * kDHead);
  const int j = (int)(row % p.nk), b = (int)(row / p.nk);
  const bool live = j < ex_batch_row(p, b).klen;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* from = (which ? p.part_dv : p.part_dk) + e;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live)
      for (int s = 0; s < p.kv_splits; ++s) {
        const float4 x = *reinterpret_cast<const float4*>(from + s * all);
        o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
      }
    const float scale = which ? 1.f : p.scale;
    const ExactOut& t = which ? p.dV : p.dK;
    ex_store4(static_cast<T*>(t.data) + b * t.batch + j * t.row + col,
              make_float4(o.x * scale, o.y * scale, o.z * scale, o.w * scale));
  }
}

// bf16 in blocks of 128 rows where the blocks of 32 are more than the CUs, or, in a long loop, which is all a
// block of 128 has on a CU then, twice as many (backward pass, 12 heads: 4 x 256 tokens, 384 blocks of 32,
// 22.3 against 20.0 us; 2 x 512 26.1 and 28.8; 1 x 1024 34.5 and 45.5; 2 x 256, 192 blocks, 15.1 and 19.8).
bool in_tiles(const ExactParams& p, int64_t blocks, int loop) {
  return p.bf16 && blocks > (loop > 384 ? 2 : 1) * (int64_t)device_cus();
}
bool dq_in_tiles(const ExactParams& p) { return in_tiles(p, exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B, p.nk); }
// And where a block of 32 keys would have a long way over the queries of its heads (64 tiles), which blocks of
// 128 keys then share (exact_kv_splits): backward pass, 1 x 16384 tokens, 1 head, 335 against 295 us; 1 x 4096, 8
// heads on 2, 158 and 149; 1 x 8192, 1 head, and 2 x 1024, 16 on 2, as long either way; 1 x 2048, 4 heads, 64 tiles,
// 35 and 46. (Where the blocks of 32 leave CUs without one it takes longer: 1 x 4096, 2 heads on 1, 58 and 64.)
bool dkv_in_tiles(const ExactParams& p) {
  return in_tiles(p, (int64_t)((p.nk + 31) / 32) * p.Hk * p.B, p.G * p.nq) || (p.bf16 && (int64_t)p.G * ((p.nq + 31) / 32) > 64);
}

// k_exact_dkv_tiles with the keys around a window's global one in blocks of their own; not for few queries or keys,
// whose way is short.
bool dkv_global_apart(const ExactParams& p) { return p.window && !few(p); }

int dkv_waves(const ExactParams& p) {  // of k_exact_dkv
  const int64_t tiles = (int64_t)p.G * ((p.nq + 31) / 32) / p.kv_splits;
  return p.bf16 && !few(p) && exact_eight_waves((int64_t)((p.nk + 31) / 32) * p.Hk * p.B * p.kv_splits, tiles) ? 8 : 4;
}

// The largest table (and a wave's sums along diagonals, as long) fits beside the tiles.
constexpr size_t kMaxTable = (2 * kMaxBiasDistance + 129) * 4;
static_assert(kDkvLds<float, 1, 4> + 5 * kMaxTable <= kMaxLds && kDkvLds<uint16_t, 2, 4> + 5 * kMaxTable <= kMaxLds &&
              kDkvLds<uint16_t, 2, 8> + 9 * kMaxTable <= kMaxLds && kDkvTilesLds + 5 * kMaxTable <= kMaxLds / 2, "LDS of a block");

template <bool BIAS>
size_t table_bytes(const ExactParams& p) { return BIAS ? (size_t)exact_bias_entries(p.D) * 4 : 0; }

template <bool BIAS, int W, bool FEW>
hipError_t launch_dq_of(const ExactParams& p, hipStream_t s) {
  const size_t lds = kDqLds<uint16_t, 2, W> + table_bytes<BIAS>(p) * p.Gp;
  const hipError_t e = exact_set_lds<k_exact_dq<BIAS, W, FEW>>(lds);
  if (e != hipSuccess) return e;
  const int64_t blocks = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B;
  hipLaunchKernelGGL((k_exact_dq<BIAS, W, FEW>), dim3((unsigned)blocks), dim3(64 * W), lds, s, p);
  return hipGetLastError();
}

template <bool BIAS>
hipError_t launch_dq(const ExactParams& p, hipStream_t s) {
  if (!dq_in_tiles(p)) {
    if (few(p)) return launch_dq_of<BIAS, 4, true>(p, s);
    return exact_eight_waves(exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B, (p.nk + 31) / 32) ? launch_dq_of<BIAS, 8, false>(p, s)
                                                                                                : launch_dq_of<BIAS, 4, false>(p, s);
  }
  const int64_t blocks = (int64_t)((p.nq + 127) / 128) * p.H * p.B;
  const size_t table = table_bytes<BIAS>(p);
  if (few(p)) {
    hipLaunchKernelGGL((k_exact_dq_tiles<BIAS, false, true>), dim3((unsigned)blocks), dim3(kExThreads), 6 * kTile64 + table, s, p);
  } else if (p.window && !p.causal) {
    const size_t lds = kDqLds<uint16_t, 2, 4> + table;
    const hipError_t e = exact_set_lds<k_exact_dq_tiles<BIAS, true, false>>(lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_exact_dq_tiles<BIAS, true, false>), dim3((unsigned)(blocks + p.H * p.B)), dim3(kExThreads), lds, s, p);
  } else {
    hipLaunchKernelGGL((k_exact_dq_tiles<BIAS, false, false>), dim3((unsigned)blocks), dim3(kExThreads), 6 * kTile64 + table, s, p);
  }
  return hipGetLastError();
}

// A block's tiles and its waves' sums along diagonals in LDS, then the bias tables of as many heads as fit. `blocks`
// of it, that need `least` LDS.
template <auto K, bool BIAS, int W = kExWaves>
hipError_t launch_dkv_kernel(const ExactParams& p, int64_t blocks, size_t base, hipStream_t s, size_t least = 0) {
  const size_t table = table_bytes<BIAS>(p);
  base += W * table;
  int heads = p.G;
  if constexpr (BIAS) {
    const size_t room = std::max(base + table, least) <= kMaxLds / 2 ? kMaxLds / 2 : kMaxLds;  // two blocks to a CU, or one
    heads = (int)std::min<size_t>(heads, (room - base) / table);
  }
  const size_t lds = std::max(base + table * heads, least);
  const hipError_t e = exact_set_lds<K>(lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(K, dim3((unsigned)blocks), dim3(64 * W), lds, s, p, heads);
  return hipGetLastError();
}
// Blocks of `keys` keys.
int64_t dkv_blocks(const ExactParams& p, int keys) { return (int64_t)((p.nk + keys - 1) / keys) * p.Hk * p.B * p.kv_splits; }

template <bool BIAS, int W, bool FEW>
hipError_t launch_dkv_of(const ExactParams& p, hipStream_t s) {
  return launch_dkv_kernel<k_exact_dkv<BIAS, W, FEW>, BIAS, W>(p, dkv_blocks(p, 32), kDkvLds<uint16_t, 2, W>, s);
}
template <bool BIAS>
hipError_t launch_dkv(const ExactParams& p, hipStream_t s) {
  if (!dkv_in_tiles(p)) {
    if (few(p)) return launch_dkv_of<BIAS, 4, true>(p, s);
    return dkv_waves(p) == 8 ? launch_dkv_of<BIAS, 8, false>(p, s) : launch_dkv_of<BIAS, 4, false>(p, s);
  }
  const int64_t blocks = dkv_blocks(p, 128);
  if (dkv_global_apart(p))
    return launch_dkv_kernel<k_exact_dkv_tiles<BIAS, true, false>, BIAS>(p, blocks + (int64_t)p.Hk * p.B, kDkvLds<uint16_t, 2, 4>, s);
  if (few(p)) return launch_dkv_kernel<k_exact_dkv_tiles<BIAS, false, true>, BIAS>(p, blocks, kDkvTilesLds, s);
  return launch_dkv_kernel<k_exact_dkv_tiles<BIAS, false, false>, BIAS>(p, blocks, kDkvTilesLds, s);
}

template <bool BIAS>
hipError_t launch_f32(const ExactParams& p, hipStream_t s) {
  const int64_t rows = ((int64_t)p.B * p.nq * p.H + kExThreads / 16 - 1) / (kExThreads / 16);
  hipLaunchKernelGGL(k_exact_stats, dim3((unsigned)rows), dim3(kExThreads), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_dkv_kernel<k_exact_backward_f32<BIAS>, BIAS>(p, dkv_blocks(p, 32) + exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B,
                                                            kDkvLds<float, 1, 4>, s, kDqLds<float, 1, 4> + table_bytes<BIAS>(p) * p.Gp);
}

template <typename T, bool BIAS>
hipError_t launch_backward(const ExactParams& p, hipStream_t s) {
  hipError_t e;
  if constexpr (ExFmt<T>::ES == 2) {
    if (!BIAS && exact_backward_small(p)) {
      const int rows = exact_small_rows(p), lds = rows * (4 * 128 + 8);  // the matrices, where S and dP start
      const bool f = few(p);
      e = f ? exact_set_lds<k_exact_backward_small<true>>(lds) : exact_set_lds<k_exact_backward_small<false>>(lds);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(f ? k_exact_backward_small<true> : k_exact_backward_small<false>, dim3((unsigned)(p.H * p.B)),
                         dim3(2 * rows), lds, s, p);
      return hipGetLastError();
    }
    if ((e = launch_dq<BIAS>(p, s)) == hipSuccess) e = launch_dkv<BIAS>(p, s);
  } else {
    e = launch_f32<BIAS>(p, s);
  }
  if (e != hipSuccess) return e;
  const int sums = BIAS ? (p.buckets * p.H + kExWaves - 1) / kExWaves : 0;
  const int64_t rows = p.kv_splits > 1 ? ((int64_t)p.B * p.nk * p.Hk * (kDHead / 4) + kExThreads - 1) / kExThreads : 0;
  if (sums + rows == 0) return hipSuccess;
  hipLaunchKernelGGL((k_exact_join_grads<T>), dim3((unsigned)(sums + rows)), dim3(kExThreads), 0, s, p, sums);
  return hipGetLastError();
}

}  // namespace

// Blocks that share a key's queries: where they leave CUs without one (few keys, or few key heads with
// many query heads), as many as that takes, of sixteen tiles of 64 at least, or a tile of 32 to a wave
// where that saves more than the join takes.
int exact_kv_splits(const ExactParams& p) {
  const bool big = dkv_in_tiles(p);
  if ((big && dkv_global_apart(p)) || exact_backward_small(p)) return 1;
  const int64_t blocks = (int64_t)((p.nk + (big ? 127 : 31)) / (big ? 128 : 32)) * p.Hk * p.B;
  const int64_t tiles = (int64_t)p.G * ((p.nq + (big ? 63 : 31)) / (big ? 64 : 32));
  const int64_t n = std::min((big ? 2 : 1) * device_cus() / blocks, tiles / (big ? 16 : kExWaves));
  return n > 1 && (big || exact_worth(tiles, n, p.bf16 ? 2 : 8)) ? (int)n : 1;
}

int64_t exact_bias_parts(const ExactParams& p) {  // a part per wave of k_exact_dkv
  if (!dkv_in_tiles(p)) return (int64_t)p.kv_splits * p.B * ((p.nk + 31) / 32) * dkv_waves(p);
  return (int64_t)p.B * (p.kv_splits * ((p.nk + 127) / 128) + (dkv_global_apart(p) ? 1 : 0)) * kExWaves;
}

ExactKernel exact_dq_kernel(const ExactParams& p) {
  return exact_backward_small(p) ? ExactKernel::kShort : dq_in_tiles(p) ? ExactKernel::kRows128 : ExactKernel::kRows32;
}
ExactKernel exact_dkv_kernel(const ExactParams& p) {
  return exact_backward_small(p) ? ExactKernel::kShort : dkv_in_tiles(p) ? ExactKernel::kRows128 : ExactKernel::kRows32;
}

hipError_t launch_exact_backward(const ExactParams& p, hipStream_t s) {
  if (p.bf16) return p.table ? launch_backward<uint16_t, true>(p, s) : launch_backward<uint16_t, false>(p, s);
  return p.table ? launch_backward<float, true>(p, s) : launch_backward<float, false>(p, s);
}

}  // namespace mca
