// Exact attention, forward: Y_h = softmax(scale Q_h K_h^T + bias) V_h with the row log-sum-exp.
//
// One pass over the keys with a running maximum m and sum l of each query's row: for a tile of 32
// keys, x = logits in base-2 units, m' = max(m, max x), P = exp2(x - m'), l' = l 2^(m - m') + sum P,
// y' = y 2^(m - m') + P V; Y = y / l and the log-sum-exp ln 2 (m + log2 l) at the end. The scores come
// as S^T = K Q^T, so that a lane holds one query's scores: m, l and the rescaling are per lane, and
// P feeds Y^T = V^T P^T from the registers it is in.
#include "exact_device.h"

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
// once for them. The key tiles are dealt out to the block's four waves and to `splits` blocks; a
// wave loads its own tiles straight into LDS ahead of their use and waits for nobody until the
// end, where the waves' states (and the blocks', in k_exact_join) are joined in a fixed order.
template <typename T> constexpr int kRowStages = ExFmt<T>::ES == 2 ? 3 : 2;
template <typename T> constexpr int kRowLds = kExWaves * kRowStages<T> * 2 * tile_bytes<T>();

template <typename T, bool BIAS>
__global__ __launch_bounds__(kExThreads) void k_exact_rows(ExactParams p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int ES = ExFmt<T>::ES, ST = kRowStages<T>, TB = tile_bytes<T>();
  float* tb = reinterpret_cast<float*>(smem + kRowLds<T>);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, hf = lane >> 5;
  const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp;
  int bid = blockIdx.x;
  const int vt = bid % nvt;
  bid /= nvt;
  const int hx = bid % Hx;
  bid /= Hx;
  const int b = bid % p.B, split = bid / p.B;
  const ExRow0 br = ex_batch_row(p, b);
  const int hk = hx * p.Gp / p.G;

  const int v = vt * 32 + c, i = v / p.Gp, g = v % p.Gp, head = hx * p.Gp + g;
  const bool live = i < br.qlen;
  const int imin = vt * 32 / p.Gp, imax = min((vt * 32 + 31) / p.Gp, br.qlen - 1);
  const int pmin = br.pos + imin, pmax = br.pos + imax;
  const ExTiles tiles = imax >= imin ? ex_key_tiles(p, pmin, pmax, br.klen) : ExTiles{-1, 0, 0};

  const char* Kb = static_cast<const char*>(p.K.data) + (b * p.K.batch + hk * kDHead) * ES;
  const char* Vb = static_cast<const char*>(p.V.data) + (b * p.V.batch + hk * kDHead) * ES;
  const uint32_t lds = lds_addr(smem) + (uint32_t)wave * ST * 2 * TB;
  const int step = kExWaves * p.splits;
  auto load = [&](int idx, int slot) __attribute__((always_inline)) {  // past the last tile: zeros
    const int k0 = ex_tile_at(tiles, idx) * 32, limit = idx < tiles.n ? br.klen : 0;
    ex_load_tile<T>(ex_rsrc(Kb, p.K.row * ES, k0, limit, ExFmt<T>::RB), (int)p.K.row * ES, lds + slot * 2 * TB, lane);
    ex_load_tile<T>(ex_rsrc(Vb, p.V.row * ES, k0, limit, ExFmt<T>::RB), (int)p.V.row * ES, lds + slot * 2 * TB + TB,
                    lane);
  };
  const int idx0 = split * kExWaves + wave;
#pragma unroll
  for (int k = 0; k < ST - 1; ++k) load(idx0 + k * step, k);

  const char* qrow = static_cast<const char*>(p.Q.data) + (b * p.Q.batch + i * p.Q.row + head * kDHead) * ES;
  const ExRow<T> q = live ? ex_global_row<T>(qrow, hf) : ex_zero_row<T>();
  const int pos = br.pos + i;
  const ExSpan keys = ex_keys_of(p, pos, br.klen);
  const float* tl = nullptr;
  if constexpr (BIAS) {
    ex_fill_bias<T>(p, tb, hx * p.Gp, p.Gp);
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
      const int side = ex_bias_side(p, k0, pmin, br.pos + (vt * 32 + 31) / p.Gp);
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
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = ex_in(keys, k0 + 4 * hf + (r & 3) + 8 * (r >> 2)) ? x[r] : -INFINITY;
    }
    ex_softmax_step(s, x);
    ex_cols_product<T>(s.y, kt + TB, x, lane);
    slot = slot == ST - 1 ? 0 : slot + 1;
  }
  s.l += ex_other_half(s.l);
  wait_vmcnt<0>();  // no load is under way into what is written next
  __syncthreads();
  // states of the waves in LDS: [wave][row][68] sums, [wave][row] (m, l)
  constexpr int YS = kDHead + 4;
  float* ys = reinterpret_cast<float*>(smem);
  float2* ml = reinterpret_cast<float2*>(smem + kExWaves * 32 * YS * 4);
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<float4*>(ys + (wave * 32 + c) * YS + 32 * cc + 8 * (r >> 2) + 4 * hf) =
          make_float4(s.y[cc][r], s.y[cc][r + 1], s.y[cc][r + 2], s.y[cc][r + 3]);
  if (hf == 0) ml[wave * 32 + c] = make_float2(s.m, s.l);
  __syncthreads();
  // thread: row tid / 8, columns 8 (tid % 8) .. + 7
  const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
  float M = -INFINITY, L = 0.f, w[kExWaves], y[8];
#pragma unroll
  for (int k = 0; k < kExWaves; ++k) M = fmaxf(M, ml[k * 32 + row].x);
  const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int k = 0; k < kExWaves; ++k) {
    w[k] = ex_exp2(ml[k * 32 + row].x - ref);
    L += ml[k * 32 + row].y * w[k];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = 0.f;
#pragma unroll
    for (int k = 0; k < kExWaves; ++k) y[e] += ys[(k * 32 + row) * YS + col + e] * w[k];
  }
  const int vr = vt * 32 + row, ir = vr / p.Gp, hr = hx * p.Gp + vr % p.Gp;
  if (ir >= br.qlen) L = 0.f;  // a padded query
  if (p.splits > 1) {
    const int64_t R = ((int64_t)(split * p.B + b) * Hx + hx) * nvt * 32 + vr;
    float4* o = reinterpret_cast<float4*>(p.part_y + R * kDHead + col);
    o[0] = make_float4(y[0], y[1], y[2], y[3]);
    o[1] = make_float4(y[4], y[5], y[6], y[7]);
    if ((threadIdx.x & 7) == 0) p.part_ml[R] = make_float2(M, L);
    return;
  }
  if (ir >= p.nq) return;
  const float inv = L > 0.f ? 1.f / L : 0.f;  // a row without keys is 0
  T* o = static_cast<T*>(p.Yo.data) + b * p.Yo.batch + ir * p.Yo.row + hr * kDHead + col;
  if constexpr (ES == 2) {
    *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv),
                                              pack_bf16x2(y[4] * inv, y[5] * inv), pack_bf16x2(y[6] * inv, y[7] * inv));
  } else {
    reinterpret_cast<float4*>(o)[0] = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    reinterpret_cast<float4*>(o)[1] = make_float4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv);
  }
  if ((threadIdx.x & 7) == 0)
    p.lse[((int64_t)b * p.H + hr) * p.nq + ir] = L > 0.f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

// Joins the parts of a row: a wave per (query, head) row, a lane per column.
template <typename T>
__global__ __launch_bounds__(kExThreads) void k_exact_join(ExactParams p) {
  const int lane = threadIdx.x & 63;
  const int nvt = (int)((p.nq * p.Gp + 31) / 32), Hx = p.H / p.Gp;
  const int64_t R = (int64_t)blockIdx.x * kExWaves + (threadIdx.x >> 6), rows = (int64_t)p.B * Hx * nvt * 32;
  const int vr = (int)(R % (nvt * 32)), i = vr / p.Gp;
  const int64_t bh = R / (nvt * 32);
  if (R >= rows || i >= p.nq) return;
  const int b = (int)(bh / Hx), h = (int)(bh % Hx) * p.Gp + vr % p.Gp;
  float M = -INFINITY, L = 0.f, y = 0.f;
  for (int s = 0; s < p.splits; ++s) M = fmaxf(M, p.part_ml[s * rows + R].x);
  const float ref = M == -INFINITY ? 0.f : M;
  for (int s = 0; s < p.splits; ++s) {
    const float2 ml = p.part_ml[s * rows + R];
    const float w = ex_exp2(ml.x - ref);
    L += ml.y * w;
    y += p.part_y[(s * rows + R) * kDHead + lane] * w;
  }
  y *= L > 0.f ? 1.f / L : 0.f;
  T* o = static_cast<T*>(p.Yo.data) + b * p.Yo.batch + i * p.Yo.row + h * kDHead + lane;
  if constexpr (ExFmt<T>::ES == 2) *o = (T)f32_to_bf16_bits(y);
  else *o = y;
  if (lane == 0) p.lse[((int64_t)b * p.H + h) * p.nq + i] = L > 0.f ? (M + __builtin_amdgcn_logf(L)) * kLn2 : -INFINITY;
}

template <typename T, bool BIAS>
hipError_t launch_rows(const ExactParams& p, hipStream_t s) {
  const size_t lds = kRowLds<T> + (BIAS ? (size_t)p.Gp * exact_bias_entries(p.D) * 4 : 0);
  hipError_t e = hipFuncSetAttribute((const void*)k_exact_rows<T, BIAS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int64_t rows = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B;
  hipLaunchKernelGGL((k_exact_rows<T, BIAS>), dim3((unsigned)(rows * p.splits)), dim3(kExThreads), lds, s, p);
  if ((e = hipGetLastError()) != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((k_exact_join<T>), dim3((unsigned)(rows * 32 / kExWaves)), dim3(kExThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

// Heads side by side in the kernels of 32 rows: a key head's whole group, unless its bias tables (and,
// backward, their gradients: two arrays per wave) do not fit beside the tiles.
int exact_group(const ExactParams& p, bool backward) {
  if (!p.table) return p.G;
  const int64_t floats = (int64_t)p.G * exact_bias_entries(p.D) * (backward ? 1 + 2 * kExWaves : 1);
  return floats <= 8192 ? p.G : 1;
}

// Blocks that share a row's keys: as many as fill the card four times over, where every wave still
// gets four tiles.
int exact_splits(const ExactParams& p) {
  const int64_t rows = exact_row_tiles(p.nq, p.Gp) * (p.H / p.Gp) * p.B, tiles = (p.nk + 31) / 32;
  const int64_t want = (4 * 256 + rows - 1) / rows, most = tiles / (4 * kExWaves);
  return (int)(want < most ? (want < 1 ? 1 : want) : (most < 1 ? 1 : most));
}

hipError_t launch_exact_forward(const ExactParams& p, hipStream_t s) {
  if (p.bf16) return p.table ? launch_rows<uint16_t, true>(p, s) : launch_rows<uint16_t, false>(p, s);
  return p.table ? launch_rows<float, true>(p, s) : launch_rows<float, false>(p, s);
}

}  // namespace mca
