// Exact attention, forward: Y_h = softmax(scale Q_h K_h^T + bias) V_h with the row log-sum-exp.
//
// One pass over the keys with a running maximum m and sum l of each query's row: for a tile of 32
// keys, x = logits in base-2 units, m' = max(m, max x), P = exp2(x - m'), l' = l 2^(m - m') + sum P,
// y' = y 2^(m - m') + P V; Y = y / l and the log-sum-exp ln 2 (m + log2 l) at the end. The scores come
// as S^T = K Q^T, so that a lane holds one query's scores: m, l and the rescaling are per lane, and
// P feeds Y^T = V^T P^T from the registers it is in.
#include <algorithm>
#include "exact_device.h"
#include "mca_kernels.h"

namespace mca {
namespace {

// A query's running statistics and its sums of P V: y[cc][r] is column 32 cc + (r & 3) + 8 (r >> 2) + 4 hf.
struct ExState {
  float m, l;  // l: of the lane's own keys
  f32x16_t y[2];
};

// x: a tile's logits (base-2 units, -inf where masked) of the lane's query; -> P in place.
__device__ __forceinline__ void ex_softmax_step(ExState& s, f32x16_t& x) {
  float t = x[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) t = fmaxf(t, x[r]);
  t = fmaxf(t, ex_other_half(t));
  const float m = fmaxf(s.m, t);
  const float ref = m == -INFINITY ? 0.f : m;  // no key yet: every P is exp2(-inf) = 0
  if (__any(m > s.m)) {
    const float a = ex_exp2(s.m - ref);
    s.l *= a;
#pragma unroll
    for (int cc = 0; cc < 2; ++cc)
#pragma unroll
      for (int r = 0; r < 16; ++r) s.y[cc][r] *= a;
  }
  s.m = m;
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    x[r] = ex_exp2(x[r] - ref);
    sum += x[r];
  }
  s.l += sum;
}

// ------------------------------------------------------------------ 32 rows per block
// Blocks of 32 (query, head) rows: a key head's Gp query heads side by side, so that the keys are read
// once for them. The key tiles are dealt out to the block's waves and to `splits` blocks; a
// wave loads its own tiles straight into LDS ahead of their use and waits for nobody until the
// end, where the waves' states (and the blocks', in k_exact_join) are joined in a fixed order.
template <typename T, int ST, int W> constexpr int kRowLds = W * ST * 2 * tile_bytes<T>();

// ST: tiles in LDS per wave, all but one of them on their way. W: waves of the block.
template <typename T, bool BIAS, int ST, int W, bool FEW>
__device__ __forceinline__ void ex_rows_block(const ExactParams& p, char* smem, int vt, int hx, int b, int split, int splits,
                                              int Gp) {
  constexpr int ES = ExFmt<T>::ES, TB = tile_bytes<T>();
  float* tb = reinterpret_cast<float*>(smem + kRowLds<T, ST, W>);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5;
  const int nvt = (int)((p.nq * Gp + 31) / 32), Hx = p.H / Gp;
  const ExRow0 br = ex_batch_row(p, b);
  const int hk = hx * Gp / p.G;

  const int v = vt * 32 + c, i = v / Gp, g = v % Gp, head = hx * Gp + g;
  const bool live = i < br.qlen;
  const int imin = vt * 32 / Gp, imax = min((vt * 32 + 31) / Gp, br.qlen - 1);
  const int pmin = br.pos + imin, pmax = br.pos + imax;
  const ExTiles tiles = imax >= imin ? ex_key_tiles(p, pmin, pmax, br.klen) : ExTiles{-1, 0, 0};

  const char* Kb = static_cast<const char*>(p.K.data) + (b * p.K.batch + hk * kDHead) * ES;
  const char* Vb = static_cast<const char*>(p.V.data) + (b * p.V.batch + hk * kDHead) * ES;
  const uint32_t lds = lds_addr(smem) + (uint32_t)wave * ST * 2 * TB;
  const int step = W * splits;
  auto load = [&](int idx, int slot) __attribute__((always_inline)) {  // past the last tile: zeros
    const int k0 = ex_tile_at(tiles, idx) * 32, limit = idx < tiles.n ? br.klen : 0;
    ex_load_tile<T>(ex_rsrc(Kb, p.K.row * ES, k0, limit, ExFmt<T>::RB), (int)p.K.row * ES, lds + slot * 2 * TB, lane);
    ex_load_tile<T>(ex_rsrc(Vb, p.V.row * ES, k0, limit, ExFmt<T>::RB), (int)p.V.row * ES, lds + slot * 2 * TB + TB,
                    lane);
  };
  const int idx0 = split * W + wave;
#pragma unroll
  for (int k = 0; k < ST - 1; ++k) load(idx0 + k * step, k);

  const char* qrow = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + head * kDHead) * ES;
  const ExRow<T> q = live ? ex_global_row<T>(qrow, hf) : ex_zero_row<T>();
  const int pos = br.pos + i;
  const ExSpan keys = ex_keys_of(p, pos, br.klen);
  const float* tl = nullptr;
  if constexpr (BIAS) {
    ex_fill_bias<T>(p, tb, hx * Gp, Gp);
    __syncthreads();
    tl = tb + g * (2 * p.D + 129) + p.D + 64;
  }
  ExState s;
  s.m = -INFINITY;
  s.l = 0.f;
  s.y[0] = s.y[1] = ex_zero16();

  int slot = 0;
  for (int idx = idx0; idx < tiles.n; idx += step) {
    wait_lds();  // the tile read last is overwritten by the next loads
    load(idx + (ST - 1) * step, slot == 0 ? ST - 1 : slot - 1);
    wait_vmcnt<(ST - 1) * 2 * ExFmt<T>::NL>();
    asm volatile("" ::: "memory");
    const char* kt = smem + (wave * ST + slot) * 2 * TB;
    const int k0 = ex_tile_at(tiles, idx) * 32;
    f32x16_t x = ex_rows_product<T>(kt, q, c, hf);
    if constexpr (BIAS) {
      const int side = ex_bias_side(p, k0, pmin, br.pos + (vt * 32 + 31) / Gp);
      if (side != 0) {
        const float far = tl[side * p.D];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, far);
      } else {
        const float* at = tl + (k0 + 4 * hf - pos);
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = __fmaf_rn(x[r], p.s2, at[(r & 3) + 8 * (r >> 2)]);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= p.s2;
    }
    if (!ex_whole(p, pmin, pmax, k0, br.klen)) {
      ex_mask(x, keys, k0 + 4 * hf, k0 > 0);
    }
    ex_softmax_step(s, x);
    ex_cols_product<T, FEW>(s.y, kt + TB, x, lane);
    slot = slot == ST - 1 ? 0 : slot + 1;
  }
  s.l += ex_other_half(s.l);
  wait_vmcnt<0>();  // no load is under way into what is written next
  __syncthreads();
  // states of the waves in LDS: [wave][row][68] sums, [wave][row] (m, l)
  constexpr int YS = kDHead + 4;
  float* ys = reinterpret_cast<float*>(smem);
  float2* ml = reinterpret_cast<float2*>(smem + W * 32 * YS * 4);
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<float4*>(ys + (wave * 32 + c) * YS + 32 * cc + 8 * (r >> 2) + 4 * hf) =
          make_float4(s.y[cc][r], s.y[cc][r + 1], s.y[cc][r + 2], s.y[cc][r + 3]);
  if (hf == 0) ml[wave * 32 + c] = make_float2(s.m, s.l);
  __syncthreads();
  // thread: 4 columns of a row, or of two
#pragma unroll
  for (int half = 0; half < 8 / W; ++half) {
    const int row = (threadIdx.x >> 4) + half * 4 * W, col = (threadIdx.x & 15) * 4;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) M = fmaxf(M, ml[k * 32 + row].x);
    const float ref = M == -INFINITY ? 0.f : M;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float w = ex_exp2(ml[k * 32 + row].x - ref);
      L += ml[k * 32 + row].y * w;
      const float4 t = *reinterpret_cast<const float4*>(ys + (k * 32 + row) * YS + col);
      y.x += t.x * w, y.y += t.y * w, y.z += t.z * w, y.w += t.w * w;
    }
    const int vr = vt * 32 + row, ir = vr / Gp, hr = hx * Gp + vr % Gp;
    if (ir >= br.qlen) L = 0.f;  // a padded query
    if (ir >= p.nq) continue;
    if (splits > 1) {
      const int64_t R = ((int64_t)(split * p.B + b) * Hx + hx) * nvt * 32 + vr;
      *reinterpret_cast<float4*>(p.part_y + R * kDHead + col) = y;
      if ((threadIdx.x & 15) == 0) p.part_ml[R] = make_float2(M, L);
    } else {
      const float inv = L > 0.f ? 1.f / L : 0.f;  // a row without keys is 0
      T* o = static_cast<T*>(p.Yo.data) + b * p.Yo.batch + ir * p.Yo.row + hr * kDHead + col;
      if (L == 0.f) y = make_float4(0.f, 0.f, 0.f, 0.f);
      if constexpr (ES == 2) *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
      else *reinterpret_cast<float4*>(o) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
      if ((threadIdx.x & 15) == 0)
        p.lse[((int64_t)b * p.H + hr) * p.nq + ir] = L > 0.f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
    }
  }
}

template <typename T, bool BIAS, int ST, int W, bool FEW>
__global__ __launch_bounds__(64 * W) void k_exact_rows(ExactParams p) {
  extern __shared__ __align__(16) char smem[];
  const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp;
  int bid = blockIdx.x;
  const int vt = bid % nvt;
  bid /= nvt;
  const int hx = bid % Hx;
  bid /= Hx;
  ex_rows_block<T, BIAS, ST, W, FEW>(p, smem, vt, hx, bid % p.B, bid / p.B, p.splits, p.Gp);
}

// Joins the parts (at most 64) of a (query, head) row: a wave per row, a lane per part for the weights and per
// column for the sums.
template <typename T>
__global__ __launch_bounds__(kExThreads) void k_exact_join(ExactParams p) {
  const int lane = threadIdx.x & 63, nv = p.nq * p.Gp, nvt = (nv + 31) / 32, Hx = p.H / p.Gp;
  const int64_t e = (int64_t)blockIdx.x * kExWaves + (threadIdx.x >> 6), rows = (int64_t)p.B * Hx * nvt * 32;
  if (e >= (int64_t)p.B * Hx * nv) return;
  const int v = (int)(e % nv), i = v / p.Gp;
  const int64_t bh = e / nv, R = bh * nvt * 32 + v;
  const int b = (int)(bh / Hx), h = (int)(bh % Hx) * p.Gp + v % p.Gp;
  const float2 ml = lane < p.splits ? p.part_ml[lane * rows + R] : make_float2(-INFINITY, 0.f);
  const float M = wave_max(ml.x), w = ex_exp2(ml.x - (M == -INFINITY ? 0.f : M));
  float L = ml.y * w;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o);
  float y = 0.f;
  for (int s0 = 0; s0 < p.splits; s0 += 8) {  // eight loads under way; parts past the last have weight 0
    float t[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) t[k] = p.part_y[(min(s0 + k, p.splits - 1) * rows + R) * kDHead + lane];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      y += t[k] * __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), s0 + k));
  }
  y = L > 0.f ? y * (1.f / L) : 0.f;
  T* o = static_cast<T*>(p.Yo.data) + b * p.Yo.batch + i * p.Yo.row + h * kDHead + lane;
  if constexpr (ExFmt<T>::ES == 2) *o = (T)f32_to_bf16_bits(y);
  else *o = y;
  if (lane == 0) p.lse[((int64_t)b * p.H + h) * p.nq + i] = L > 0.f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

// ------------------------------------------------------------------ up to 128 queries and keys, bf16
// For grids that fill the card: a block has a (batch row, head)'s K and V in LDS, a wave for each 32 of its queries,
// which puts more short rows on a CU than blocks of 128 queries do (300 x 40 tokens, 16 heads, 20 and 35 us; 64 x
// 64, 12 heads, 7.0 and 8.3; 64 rows of 16 to 128 10.7 and 11.0; 128 x 128, 101 MB, 22.3 and 22.4, of which P's
// second products are 3).
__global__ __launch_bounds__(kExThreads) void k_exact_forward_small(ExactParams p) {
  using T = uint16_t;
  extern __shared__ __align__(16) char smem[];  // K, V
  const int M = exact_small_rows(p) * 128;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5, h = blockIdx.x % p.H, b = blockIdx.x / p.H, r0 = 32 * wave, i = r0 + c;
  const ExRow0 br = ex_batch_row(p, b);
  const int64_t hcol = h * kDHead;
  auto load = [&](const ExactRows& m, uint32_t to) __attribute__((always_inline)) {
    const char* base = static_cast<const char*>(m.data) + (b * m.batch + h / p.G * kDHead) * 2;
    ex_load_tile<T>(ex_rsrc(base, m.row * 2, r0, br.klen, 128), (int)m.row * 2, lds_addr(smem) + to + 4096u * wave, lane);
  };
  load(p.K, 0);
  load(p.V, M);
  const char* qrow = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + hcol) * 2;
  const ExRow<T> q = i < br.qlen ? ex_global_row<T>(qrow, hf) : ex_zero_row<T>();
  wait_vmcnt<0>();
  __syncthreads();

  ExState s;
  s.m = -INFINITY;
  s.l = 0.f;
  s.y[0] = s.y[1] = ex_zero16();
  const int last = min(r0 + 32, br.qlen) - 1;
  if (last >= r0) {  // wave-uniform
    const ExTiles tiles = ex_key_tiles(p, br.pos + r0, br.pos + last, br.klen);
    const ExSpan keys = ex_keys_of(p, br.pos + i, br.klen);
#pragma clang loop unroll(disable)
    for (int t = 0; t < tiles.n; ++t) {
      const int kt = ex_tile_at(tiles, t), k0 = 32 * kt;
      f32x16_t x = ex_rows_product<T>(smem + 4096 * kt, q, c, hf);
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= p.s2;
      if (!ex_whole(p, br.pos + r0, br.pos + last, k0, br.klen)) ex_mask(x, keys, k0 + 4 * hf, k0 > 0);
      ex_softmax_step(s, x);
      ex_cols_product<T, true>(s.y, smem + M + 4096 * kt, x, lane);
    }
  }
  s.l += ex_other_half(s.l);
  const float L = i < br.qlen ? s.l : 0.f;
  if (L == 0.f) s.y[0] = s.y[1] = ex_zero16();
  if (hf == 0 && i < p.nq)
    p.lse[((int64_t)b * p.H + h) * p.nq + i] = L > 0.f ? (s.m + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
  __syncthreads();
  char* out = static_cast<char*>(p.Yo.data) + (b * p.Yo.batch + (int64_t)r0 * p.Yo.row + hcol) * 2;
  ex_store_rows32(smem + wave * 32 * 144, s.y, L > 0.f ? 1.f / L : 0.f, out, p.Yo.row * 2, p.nq - r0, lane);
}

// ------------------------------------------------------------------ 128 or 256 queries per block, bf16
// Four waves of 32 MT queries of one head share key tiles of 64. What bounds it is issue on each
// SIMD, as in the output pass of the sampled layer: a half tile of 32 keys runs as slots that are
// fixed in the source, each one MFMA (in turn S of half tile h + 1 and P V of h - 1) beside the vector
// work of two scores of h, and reloads the fragment that its MFMA has used. K and V tiles are
// loaded straight into LDS, three buffers each.
//
// No running maximum: P = exp2(x - M) under M, the largest logit of the row's first 32 keys, needs no
// correction of what has been summed, and keeps its relative precision, in bf16 too, up to the
// type's range. A row whose sum passes 2^64 (logits 44 above M), or whose first keys the bias all
// masked and whose sum is below 2^-20, has its block take the pass again with a running maximum.
//
// FEW: as of k_exact_rows. What the rounding of P took off goes through an MFMA of its own, behind that of P V.
template <bool BIAS, int MT, bool WIN, bool FEW>
__global__ __launch_bounds__(kExThreads) __attribute__((amdgpu_waves_per_eu(MT == 1 ? 3 : 2))) void k_exact_tiles(ExactParams p) {
  constexpr int QB = 128 * MT;
  extern __shared__ __align__(16) char smem[];  // three K tiles, three V tiles, the bias table
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5;
  int qt, pair;
  const int nqt = (p.nq + QB - 1) / QB;
  int bid = blockIdx.x;
  if constexpr (WIN) {  // the first blocks: the rows around a global query
    if (bid < p.H * p.B) {
      const int first = ex_global_rows(p, ex_batch_row(p, bid / p.H));
      if (first >= 0) ex_rows_block<uint16_t, BIAS, 2, 4, false>(p, smem, first / 32, bid % p.H, bid / p.H, 0, 1, 1);
      return;
    }
    bid -= p.H * p.B;
  }
  ex_block_pair(bid, nqt, p.H * p.B, p.causal || p.window, qt, pair);
  if (p.causal) qt = nqt - 1 - qt;  // the longest rows first
  const int h = pair % p.H, b = pair / p.H, hk = h / p.G;
  const ExRow0 br = ex_batch_row(p, b);
  const int qw = qt * QB + wave * 32 * MT;  // the wave's first query
  const int global = WIN ? ex_global_rows(p, br) : -1;
  const int first = qt * QB + (WIN && global == qt * QB ? 32 : 0), last = min(qt * QB + QB, br.qlen) - 1;
  const ExTiles tiles = last >= first ? ex_key_tiles<64>(p, br.pos + first, br.pos + last, br.klen, !WIN) : ExTiles{-1, 0, 0};
  const bool mine = !WIN || qw != global;  // another block has the wave's rows
  // keys that all of the wave's queries attend
  const ExRange whole = ex_whole_keys(p, br.pos + qw, br.pos + min(qw + 32 * MT, br.qlen) - 1, br.klen);

  char* yrow = static_cast<char*>(p.Yo.data) + ((int64_t)b * p.Yo.batch + (int64_t)qw * p.Yo.row + h * kDHead) * 2;
  float* lse = p.lse + ((int64_t)b * p.H + h) * p.nq;
  const char* Kb = static_cast<const char*>(p.K.data) + (b * p.K.batch + hk * kDHead) * 2;
  const char* Vb = static_cast<const char*>(p.V.data) + (b * p.V.batch + hk * kDHead) * 2;
  const int kpitch = (int)p.K.row * 2, vpitch = (int)p.V.row * 2;
  const uint32_t kl = ex_load64(wave, lane, kpitch), vl = ex_load64<true>(wave, lane, vpitch);
  const uint32_t lds = lds_addr(smem);
  // Tile t into buffer `slot`, in the order of t; past the last tile: zeros
  ExStream ks, vs;
  auto load = [&](ExStream& m, const char* base, int pitch, int t, uint32_t off, uint32_t to) __attribute__((always_inline)) {
    if (t == 0 || (tiles.first >= 0 && t == 1)) m = ex_stream(base, pitch, ex_tile_at(tiles, t) * 64, br.klen);
    if (t >= tiles.n) m.rows = 0;
    ex_load_next64(m, pitch, off, to, wave);
  };
  auto load_k = [&](int t, int slot) __attribute__((always_inline)) { load(ks, Kb, kpitch, t, kl, lds + slot * kTile64); };
  auto load_v = [&](int t, int slot) __attribute__((always_inline)) { load(vs, Vb, vpitch, t, vl, lds + (3 + slot) * kTile64); };
  load_k(0, 0);
  ExRow<uint16_t> q[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int i = min(qw + 32 * m + c, br.qlen - 1);
    const char* row = static_cast<const char*>(p.Q.data) + ((int64_t)b * p.Q.batch + (int64_t)i * p.Q.row + h * kDHead) * 2;
    q[m] = i >= 0 ? ex_global_row<uint16_t>(row, hf) : ex_zero_row<uint16_t>();
  }
  load_k(1, 1);
  load_v(0, 0);
  float* tb = reinterpret_cast<float*>(smem + 6 * kTile64);
  const float* tl = tb + p.D + 64;
  if constexpr (BIAS) ex_fill_bias<uint16_t>(p, tb, h, 1);

  const ExRows64 ka = ex_rows64(lane);
  const ExCols64<true> va = ex_cols64<true>(lane);
  const f32x16_t zero = ex_zero16();
  f32x16_t y[MT][2], s0[MT], s1[MT];
  struct P16 {
    u32x4_t v[2], rest[FEW ? 2 : 1];
  };
  P16 pa[MT], pb[MT];  // P of a half tile, 16 keys each
  u32x4_t kf[4], vf[2][2];
  float l[MT], nm[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    y[m][0] = y[m][1] = zero;
    pb[m].v[0] = pb[m].v[1] = u32x4_t{0u, 0u, 0u, 0u};  // the first P V multiplies zeros
    if constexpr (FEW) pb[m].rest[0] = pb[m].rest[1] = pb[m].v[0];
    l[m] = 0.f;
  }
  vf[0][0] = vf[0][1] = vf[1][0] = vf[1][1] = u32x4_t{0u, 0u, 0u, 0u};

  // What a half tile's scores still need: masks and the bias of near pairs. fac, add: a logit is
  // fac * score + add.
  float fac = p.s2, add = 0.f;
  // Half tiles of which the wave's queries attend nothing, under a window: P = 0 from the addition that the
  // logits have anyway, with no masks to work out (8 x 1057 tokens, 12 heads, window 256: 26.2 and 25.0 us, 64:
  // 24.5 and 22.1; the backward pass gains nothing).
  const ExRange near{br.pos + qw - p.half - 31, min(br.pos + min(qw + 32, br.qlen) - 1 + p.half, br.klen - 1)};
  auto any = [&](int k0) __attribute__((always_inline)) { return mine && qw < br.qlen && (k0 == 0 || ex_has(near, k0)); };
  auto fix = [&](f32x16_t (&s)[MT], int k0) __attribute__((always_inline)) {
    if constexpr (WIN) {
      fac = p.s2;
      add = any(k0) ? 0.f : -INFINITY;
      if (add != 0.f) return;
    }
    if constexpr (BIAS) {
      const int side = ex_bias_side(p, k0, br.pos + qw, br.pos + qw + 32 * MT - 1);
      // 64 queries: a tile near either half has more distances than the table holds for one
      fac = p.s2;
      add = 0.f;
      if (side != 0) {
        add = tl[side * p.D];
      } else {
        fac = 1.f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int pos = br.pos + qw + 32 * m + ex_opaque(c);
          const int ms = MT == 1 ? 0 : ex_bias_side(p, k0, br.pos + qw + 32 * m, br.pos + qw + 32 * m + 31);
          if (ms != 0) {
            const float far = tl[ms * p.D];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[m][r] = __fmaf_rn(s[m][r], p.s2, far);
          } else {
            const float* at = tl + (k0 + 4 * hf - pos);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[m][r] = __fmaf_rn(s[m][r], p.s2, at[(r & 3) + 8 * (r >> 2)]);
          }
        }
      }
    }
    if (__builtin_expect(!ex_has(whole, k0), 0)) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const ExSpan keys = ex_keys_of(p, br.pos + qw + 32 * m + ex_opaque(c), br.klen);
        ex_mask(s[m], keys, k0 + 4 * hf, MT == 2 || k0 > 0);  // 256 queries: no window
      }
    }
  };
  // Half tile h: P of cur into po, S of half tile h + 1 into nxt, P V of half tile h - 1 (pi, vf); K half
  // tile h + 2 and V half tile h are `half` of the tiles at kt and vt.
  auto step = [&](f32x16_t (&cur)[MT], f32x16_t (&nxt)[MT], const P16 (&pi)[MT], P16 (&po)[MT], const char* kt, const char* vt,
                  int half) __attribute__((always_inline)) {
    float e0 = 0.f, e1 = 0.f;
#pragma unroll
    for (int j = 0; j < 8 * MT; ++j) {
      const int i = j / (2 * MT), m = (j >> 1) % MT, pp = i >> 1, cc = i & 1;
      if (j % 2 == 0) {
        nxt[m] = ex_mfma<uint16_t>(kf[i], q[m].v[i], i == 0 ? zero : nxt[m]);
        __builtin_amdgcn_sched_barrier(0);  // the reload takes the registers the MFMA has read
        if (m == MT - 1) kf[i] = ex_read_row(kt, ka, half, i);
      } else {
        y[m][cc] = ex_mfma<uint16_t>(vf[pp][cc], pi[m].v[pp], y[m][cc]);
        if constexpr (FEW) y[m][cc] = ex_mfma<uint16_t>(vf[pp][cc], pi[m].rest[pp], y[m][cc]);
        __builtin_amdgcn_sched_barrier(0);
        if (m == MT - 1) vf[pp][cc] = ex_read_col(vt, va, half, pp, cc);
      }
      const int n = j >> 3, k = j & 7;  // scores 2 k, + 1 of query tile n
      const float a = BIAS || WIN ? nm[n] + add : nm[n], f = BIAS ? fac : p.s2;
      const float x0 = __fmaf_rn(cur[n][2 * k], f, a), x1 = __fmaf_rn(cur[n][2 * k + 1], f, a);
      if (j > 0) {  // the pair before: its exp2 results are not waited for
        const int o = (j - 1) >> 3;
        l[o] += e0;
        l[o] += e1;
        uint32_t w = pack_bf16x2(e0, e1);
        ex_pin(w);
        po[o].v[((j - 1) >> 2) & 1][(j - 1) & 3] = w;
        if constexpr (FEW) po[o].rest[((j - 1) >> 2) & 1][(j - 1) & 3] = ex_pack_rest(e0, e1, w);
      }
      e0 = ex_exp2(x0);
      e1 = ex_exp2(x1);
      ex_pin(e0);
      ex_pin(e1);
      __builtin_amdgcn_sched_barrier(0);
    }
    l[MT - 1] += e0;
    l[MT - 1] += e1;
    po[MT - 1].v[1][3] = pack_bf16x2(e0, e1);
    if constexpr (FEW) po[MT - 1].rest[1][3] = ex_pack_rest(e0, e1, po[MT - 1].v[1][3]);
  };

  if constexpr (BIAS) __syncthreads();
  wait_vmcnt<4>();  // K tile 0
  stage_barrier();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x4_t k = ex_read_row(smem, ka, 0, i);
#pragma unroll
    for (int m = 0; m < MT; ++m) s0[m] = ex_mfma<uint16_t>(k, q[m].v[i], i == 0 ? zero : s0[m]);
    kf[i] = ex_read_row(smem, ka, 1, i);
  }
  fix(s0, ex_tile_at(tiles, 0) * 64);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float t = s0[m][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) t = fmaxf(t, s0[m][r]);
    t = __fmaf_rn(fmaxf(t, ex_other_half(t)), fac, add);  // fac > 0
    nm[m] = t > -INFINITY ? -t : 0.f;
  }
  int b0 = 0, b1 = 1, b2 = 2;  // buffers of tiles t, t + 1, t + 2
#pragma clang loop unroll(disable)
  for (int t = 0; t < tiles.n; ++t) {
    wait_vmcnt<0>();
    stage_barrier();
    load_k(t + 2, b2);
    load_v(t + 1, b1);
    const char *kt = smem + b1 * kTile64, *vt = smem + (3 + b0) * kTile64;
    const int k0 = ex_tile_at(tiles, t) * 64;
    if (t > 0) fix(s0, k0);
    step(s0, s1, pb, pa, kt, vt, 0);
    fix(s1, k0 + 32);
    step(s1, s0, pa, pb, kt, vt, 1);
    const int o = b0;
    b0 = b1;
    b1 = b2;
    b2 = o;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      y[m][i & 1] = ex_mfma<uint16_t>(vf[i >> 1][i & 1], pb[m].v[i >> 1], y[m][i & 1]);
      if constexpr (FEW) y[m][i & 1] = ex_mfma<uint16_t>(vf[i >> 1][i & 1], pb[m].rest[i >> 1], y[m][i & 1]);
    }
  wait_vmcnt<0>();  // no load is under way into what is written next
  bool again = false;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    l[m] += ex_other_half(l[m]);
    const bool live = qw + 32 * m + c < br.qlen && tiles.n > 0 && mine;
    again = again || (live && (!(l[m] <= 0x1p64f) || (BIAS && l[m] < 0x1p-20f)));
    if (!live) l[m] = 0.f;  // a padded query
  }
  // rows qw + 32 m on: their sums under -nmax, normalised and written
  auto store = [&](int m, float nmax, float sum, f32x16_t (&ym)[2]) __attribute__((always_inline)) {
    if (!mine) return;
    const int first = qw + 32 * m, ln = ex_opaque(lane), i = first + (ln & 31);
    if (ln < 32 && i < p.nq) lse[i] = sum > 0.f ? (__builtin_amdgcn_logf(sum) - nmax) * kLn2 : -INFINITY;
    if (sum == 0.f) ym[0] = ym[1] = zero;  // what was summed for it may be anything
    ex_store_rows32(smem + wave * 32 * 144, ym, sum > 0.f ? 1.f / sum : 0.f, yrow + (int64_t)32 * m * p.Yo.row * 2,
                    p.Yo.row * 2, p.nq - first, ln);
  };
  if (__builtin_expect(__syncthreads_or(again), 0)) {
#pragma clang loop unroll(disable)
    for (int m = 0; m < MT; ++m) {  // one after the other: the waves keep in step
      ExState s;
      s.m = -INFINITY;
      s.l = 0.f;
      s.y[0] = s.y[1] = zero;
      const int first = qw + 32 * m, ln = ex_opaque(lane), cs = ln & 31, hs = ln >> 5, pos = br.pos + first + cs;
      const ExCols64<true> vc = ex_cols64<true>(ln);
      const ExSpan keys = ex_keys_of(p, pos, br.klen);
      const char* row = static_cast<const char*>(p.Q.data) +
                        ((int64_t)b * p.Q.batch + (int64_t)min(first + cs, br.qlen - 1) * p.Q.row + h * kDHead) * 2;
      const ExRow<uint16_t> qm = ex_global_row<uint16_t>(row, hs);  // a block without queries is never here
#pragma clang loop unroll(disable)
      for (int t = 0; t < tiles.n; ++t) {
        load_k(t, 0);
        load_v(t, 0);
        wait_vmcnt<0>();
        __syncthreads();
#pragma clang loop unroll(disable)
        for (int half = 0; half < 2; ++half) {
          const int k0 = ex_tile_at(tiles, t) * 64 + 32 * half;
          f32x16_t x = ex_rows_product<uint16_t>(smem + half * 4096, qm, cs, hs);
          const int side = BIAS ? ex_bias_side(p, k0, br.pos + first, br.pos + first + 31) : 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int e = (r & 3) + 8 * (r >> 2);
            const float bias = !BIAS ? 0.f : side != 0 ? tl[side * p.D] : tl[k0 + 4 * hs - pos + e];
            x[r] = ex_in(keys, k0 + 4 * hs + e) ? __fmaf_rn(x[r], p.s2, bias) : -INFINITY;
          }
          ex_softmax_step(s, x);
#pragma unroll
          for (int pp = 0; pp < 2; ++pp) {
            u32x4_t x8, rest;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              x8[w] = pack_bf16x2(x[8 * pp + 2 * w], x[8 * pp + 2 * w + 1]);
              if constexpr (FEW) rest[w] = ex_pack_rest(x[8 * pp + 2 * w], x[8 * pp + 2 * w + 1], x8[w]);
            }
#pragma unroll
            for (int cc = 0; cc < 2; ++cc) {
              const u32x4_t v = ex_read_col(smem + 3 * kTile64, vc, half, pp, cc);
              s.y[cc] = ex_mfma<uint16_t>(v, x8, s.y[cc]);
              if constexpr (FEW) s.y[cc] = ex_mfma<uint16_t>(v, rest, s.y[cc]);
            }
          }
        }
        __syncthreads();
      }
      s.l += ex_other_half(s.l);
      store(m, -s.m, first + cs < br.qlen ? s.l : 0.f, s.y);
      __syncthreads();
    }
    return;
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) store(m, nm[m], l[m], y[m]);
}

template <bool BIAS, int MT, bool WIN, bool FEW = false>
hipError_t launch_tiles(const ExactParams& p, hipStream_t s) {
  const size_t table = BIAS ? (size_t)exact_bias_entries(p.D) * 4 : 0;
  const size_t lds = table + (WIN ? (size_t)kRowLds<uint16_t, 2, 4> : 6 * kTile64);
  const int64_t blocks = ((int64_t)((p.nq + 128 * MT - 1) / (128 * MT)) + WIN) * p.H * p.B;
  if constexpr (WIN) {
    const hipError_t e = exact_set_lds<k_exact_tiles<BIAS, MT, WIN, FEW>, 512>(lds);
    if (e != hipSuccess) return e;
  }
  static_assert(6 * kTile64 + (2 * kMaxBiasDistance + 129) * 4 <= 65536 - 512, "LDS that needs no leave");
  hipLaunchKernelGGL((k_exact_tiles<BIAS, MT, WIN, FEW>), dim3((unsigned)blocks), dim3(kExThreads), lds, s, p);
  return hipGetLastError();
}

template <typename T, bool BIAS, int ST, int W, bool FEW = false>
hipError_t launch_rows_of(const ExactParams& p, hipStream_t s) {
  const size_t lds = kRowLds<T, ST, W> + (BIAS ? (size_t)p.Gp * exact_bias_entries(p.D) * 4 : 0);
  hipError_t e = exact_set_lds<k_exact_rows<T, BIAS, ST, W, FEW>>(lds);
  if (e != hipSuccess) return e;
  const int64_t rows = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B;
  hipLaunchKernelGGL((k_exact_rows<T, BIAS, ST, W, FEW>), dim3((unsigned)(rows * p.splits)), dim3(64 * W), lds, s, p);
  if ((e = hipGetLastError()) != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((k_exact_join<T>), dim3((unsigned)(((int64_t)p.B * p.H * p.nq + kExWaves - 1) / kExWaves)), dim3(kExThreads), 0, s, p);
  return hipGetLastError();
}

// FEW of the kernels above: P is multiplied to more than the type's bits (ex_cols_product). By the lengths alone, so
// that a row's precision does not depend on how many there are: up to 128 keys, a tile to each wave of a block, or
// up to 32 queries (32 x 1 token, 16 heads on 4, up to 16384 keys, 73.2 and 73.6 us; 1 x 1, 701 keys, 7.5 and 7.9; 64
// rows of 16 to 128 tokens, 12 heads, 11.5 and 12.5).
bool few(const ExactParams& p) { return p.bf16 && (p.nk <= 128 || p.nq <= 32); }

// bf16: two tiles, 64 KB of LDS for a block, two of them to a CU. float32, whose tiles are twice as large: one, and two
// blocks to a CU, which cover each other's loads (forward, 12 heads, two tiles against one: 32 x 128 tokens 50.0 and
// 34.2 us; 2 x 320, where every block has a CU of its own, 14.7 and 14.1; 1 x 128 7.9 and 7.2; 32 x 1, 16 heads on 4,
// 16384 keys, 240 and 197).
template <typename T, bool BIAS>
hipError_t launch_rows(const ExactParams& p, hipStream_t s) {
  const int64_t blocks = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B * p.splits;
  if constexpr (ExFmt<T>::ES == 4) {
    return launch_rows_of<T, BIAS, 1, 4>(p, s);
  } else {
    const bool eight = exact_eight_waves(blocks, ((p.nk + 31) / 32) / p.splits);
    if (few(p)) return eight ? launch_rows_of<T, BIAS, 2, 8, true>(p, s) : launch_rows_of<T, BIAS, 2, 4, true>(p, s);
    return eight ? launch_rows_of<T, BIAS, 2, 8>(p, s) : launch_rows_of<T, BIAS, 2, 4>(p, s);
  }
}

}  // namespace

// Heads side by side in the kernels of 32 rows: a key head's whole group, unless its bias tables do not
// fit beside the tiles.
int exact_group(const ExactParams& p) {
  return !p.table || (int64_t)p.G * exact_bias_entries(p.D) * 4 <= (int64_t)kMaxLds - kRowLds<uint16_t, 2, 8> ? p.G : 1;
}

// bf16 in blocks of 128 queries or more, or of a whole short row: where the blocks of 32 rows are more than the CUs
// (forward, 12 heads: 8 x 128 tokens, 384 blocks of 32, 7.1 against 6.8 us; 8 x 160 7.4 and 7.1; 3 x 300 8.5 and 8.3;
// 2 x 256, 192 blocks, 6.9 and 7.5; 1 x 512 7.4 and 10.3). Long rows that are not many more blocks would still be
// faster in blocks of 32 (1 x 1024 13.6 and 16.4; 1 x 2048, 8 heads, 22.3 and 28.4). Rows of a single block of 32 over
// many keys stay: its four waves share the keys, of which a wave of the other kernel reads all.
static bool forward_in_tiles(const ExactParams& p) {
  return p.bf16 && exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B > device_cus() &&
         (p.nq * p.Gp > 32 || p.nk <= 512);
}
// 256 queries per block instead of 128 halve the LDS reads and the loads per score, and take about 1.75
// times as long: by what the CU with the most blocks has to do (4 x 4096 tokens, 12 heads: 6 blocks
// against 3, 220 and 198 us; 8 x 1057: 4 and 2, 44.7 and 39.7; 3 x 2000: 3 and 2, 55.9 and 61.1; 32 x
// 250: 3 and 2, 15.7 and 16.9). Not with a bias,
// whose table leaves too few registers, nor under a window, where a wave of fewer queries has fewer keys
// that others of the block need.
static bool forward_wide(const ExactParams& p) {
  const int64_t q128 = (p.nq + 127) / 128, pairs = (int64_t)p.H * p.B;
  return !p.table && !p.window && 4 * blocks_per_cu(q128 * pairs) > 7 * blocks_per_cu((q128 + 1) / 2 * pairs);
}

// Blocks that share a row's keys. Enough to give every CU one, of three tiles to a wave at least (float32,
// whose tiles take four times as long: less than one); or, where the keys are so long that sixteen tiles
// stay to a wave (four), up to four to a CU, which even out rows of different lengths. Not for less than
// the join takes. A token, 12 heads, bf16: 1500 keys 10.6 us in one part, 10.4 in 4, 10.0 in 8; 4000 keys
// 20.0, 12.2, 10.3; 16000 keys 72.2, 15.9 in 16; 701 keys 7.7, 10.0 in 4. 32 rows of one token, 16
// heads on 4, 2048 to 16384 keys: 65.8 us in 2 parts, 63.6 in 8, 71.8 in 32.
int exact_splits(const ExactParams& p) {
  if (forward_in_tiles(p)) return 1;
  const int64_t rows = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B, tiles = (p.nk + 31) / 32;
  const int64_t fill = std::min((device_cus() + rows - 1) / rows, tiles / (p.bf16 ? 12 : 3));
  const int64_t even = std::min(4 * device_cus() / rows, tiles / (p.bf16 ? 64 : 16));
  const int64_t n = std::min<int64_t>(std::max<int64_t>(std::max(fill, even), 1), 64);
  return exact_worth(tiles, n, p.bf16 ? 1 : 4) ? (int)n : 1;
}

// Eight waves to a block instead of four, bf16: where every block has a CU of its own and more than two tiles to
// a wave (a token, 12 heads: 1024 keys 10.0 us with four waves, 8.6 with eight, 701 keys 8.7 and 7.8, 300 keys,
// 10 tiles, 7.0 and 7.1; 2 x 1024 tokens, 4 heads, forward 10.8 and 9.1, backward 27.4 and 25.1; backward
// 2 x 256, 8 tiles, 15.1 and 17.0). Not float32, which its matrix instructions bound: 1 x 512 tokens, forward
// and backward, 74 and 72; 4 x 201, 8 heads on 2, with a bias, 59 and 61.
bool exact_eight_waves(int64_t blocks, int64_t tiles) { return tiles > 8 && blocks <= device_cus(); }

ExactKernel exact_forward_kernel(const ExactParams& p) {
  if (!forward_in_tiles(p)) return ExactKernel::kRows32;
  if (exact_small(p)) return ExactKernel::kShort;
  return !few(p) && forward_wide(p) ? ExactKernel::kRows256 : ExactKernel::kRows128;
}

hipError_t launch_exact_forward(const ExactParams& p, hipStream_t s) {
  const int rows = exact_small_rows(p);
  switch (exact_forward_kernel(p)) {
    case ExactKernel::kShort:
      hipLaunchKernelGGL(k_exact_forward_small, dim3((unsigned)(p.H * p.B)), dim3(2 * rows), rows * 256, s, p);
      return hipGetLastError();
    case ExactKernel::kRows256:
      return launch_tiles<false, 2, false>(p, s);
    case ExactKernel::kRows128:
      if (few(p)) return p.table ? launch_tiles<true, 1, false, true>(p, s) : launch_tiles<false, 1, false, true>(p, s);
      if (p.window && !p.causal) return p.table ? launch_tiles<true, 1, true>(p, s) : launch_tiles<false, 1, true>(p, s);
      return p.table ? launch_tiles<true, 1, false>(p, s) : launch_tiles<false, 1, false>(p, s);
    default:
      break;
  }
  if (p.bf16) return p.table ? launch_rows<uint16_t, true>(p, s) : launch_rows<uint16_t, false>(p, s);
  return p.table ? launch_rows<float, true>(p, s) : launch_rows<float, false>(p, s);
}

}  // namespace mca
