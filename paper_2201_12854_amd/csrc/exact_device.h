// Device side of the exact attention kernels: tiles of 32 rows in LDS, the operands read from
// them, which pairs attend, and the relative bias.
//
// Matrix products run on 32x32 MFMA tiles (bf16 32x32x16, float32 32x32x2). A lane l = 32 h + c
// of the 32x32 result holds column c of rows (r & 3) + 8 (r >> 2) + 4 h, r = 0 .. 15. The order in
// which a product runs over its inner index is free, so both operands may take it as it lies:
//   rows against rows (inner index d = 0 .. 63): lane l of either operand gives row c, 16 bytes
//     at a time: chunk 2 g + h of its row (8 bf16, one MFMA; 4 float32, four MFMAs);
//   a 32x32 result X as the second operand of a product over its rows: lane l gives its own 16
//     registers, and the first operand is read for the same rows (bf16 with the transposing LDS
//     read, float32 one element per MFMA). No data moves between the two products.
#pragma once

#include "exact.h"
#include "mca_device.h"

namespace mca {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kExThreads = 256;
constexpr int kExWaves = 4;

template <typename T> struct ExFmt;
template <> struct ExFmt<uint16_t> {  // bfloat16
  static constexpr int RB = 128;   // bytes of a tile row (64 columns)
  static constexpr int NG = 4;     // 32-byte groups of a row
  static constexpr int NL = 4;     // direct loads (1 KB each) of a tile of 32 rows
  static constexpr int ES = 2;
};
template <> struct ExFmt<float> {
  static constexpr int RB = 256;
  static constexpr int NG = 8;
  static constexpr int NL = 8;
  static constexpr int ES = 4;
};
template <typename T> constexpr int tile_bytes() { return 32 * ExFmt<T>::RB; }

// Position of 16-byte chunk c of tile row r: c ^ ex_swz(r). bf16 rows are half the LDS banks wide:
// reads of one chunk of 16 consecutive rows want the row pairs' permutations distinct, and the
// transposing reads of rows 4 k .. 4 k + 3 want those of its two row pairs to differ in bit 2: the
// pair's number with its three bits reversed. float32 rows fill the banks: one chunk of 16 rows.
template <typename T> __device__ __forceinline__ int ex_swz(int r);
template <> __device__ __forceinline__ int ex_swz<uint16_t>(int r) {
  return ((r >> 3) & 1) | ((r >> 1) & 2) | ((r << 1) & 4);
}
template <> __device__ __forceinline__ int ex_swz<float>(int r) { return r & 15; }

// ------------------------------------------------------------------ direct loads
// Descriptor of rows row0 .. row0 + 31 of a head's [*, 64] slice that ends at row `limit` (rows at
// or past it read as zeros), as four scalar words. The offsets within it stay below 2^31: the host
// refuses row pitches of 2^25 bytes or more.
__device__ __forceinline__ u32x4_t ex_rsrc(const char* base, int64_t pitch, int row0, int limit, int rowbytes) {
  const int rows = min(limit - row0, 32);
  const int bytes = rows > 0 ? (rows - 1) * (int)pitch + rowbytes : 0;
  const uint64_t a = (uint64_t)(uintptr_t)base + (uint64_t)((int64_t)row0 * pitch);
  u32x4_t w;
  w[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  w[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu));
  w[2] = (uint32_t)__builtin_amdgcn_readfirstlane(bytes);
  w[3] = 0x00020000u;  // 32-bit data format
  return w;
}

// 16 bytes per lane straight into LDS: lane l's land at lds + 16 l, zeros where out of range. The
// five wait states are those that scalar operands written by vector instructions ask for.
__device__ __forceinline__ void ex_load_lds16(u32x4_t rs, uint32_t off, uint32_t lds) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rs), "{m0}"(lds) : "memory");
}
// 4 bytes per lane.
__device__ __forceinline__ void ex_load_lds4(u32x4_t rs, uint32_t off, uint32_t lds) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(off), "s"(rs), "{m0}"(lds) : "memory");
}

// The wave's loads of a whole tile of 32 rows.
template <typename T>
__device__ __forceinline__ void ex_load_tile(u32x4_t rs, int pitch, uint32_t lds, int lane) {
  constexpr int CH = ExFmt<T>::RB / 16, RPL = 64 / CH;  // chunks per row, rows per load
#pragma unroll
  for (int n = 0; n < ExFmt<T>::NL; ++n) {
    const int row = RPL * n + lane / CH;
    ex_load_lds16(rs, (uint32_t)(row * pitch + (((lane % CH) ^ ex_swz<T>(row)) << 4)), lds + 1024u * n);
  }
}

// x, which the compiler can neither foresee nor move: what a rare branch computes from it is not kept
// in registers outside of the branch.
__device__ __forceinline__ int ex_opaque(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// ------------------------------------------------------------------ operands and products
template <typename T> struct ExRow { u32x4_t v[ExFmt<T>::NG]; };  // a lane's half of a row

template <typename T>
__device__ __forceinline__ ExRow<T> ex_zero_row() {
  ExRow<T> f;
#pragma unroll
  for (int g = 0; g < ExFmt<T>::NG; ++g) f.v[g] = u32x4_t{0u, 0u, 0u, 0u};
  return f;
}
// From memory: the row starts at `row`.
template <typename T>
__device__ __forceinline__ ExRow<T> ex_global_row(const char* row, int hf) {
  ExRow<T> f;
#pragma unroll
  for (int g = 0; g < ExFmt<T>::NG; ++g) f.v[g] = *reinterpret_cast<const u32x4_t*>(row + 32 * g + 16 * hf);
  return f;
}
// Chunk 2 g + hf of tile row c.
template <typename T>
__device__ __forceinline__ u32x4_t ex_tile_chunk(const char* tile, int c, int hf, int g) {
  return *reinterpret_cast<const u32x4_t*>(tile + c * ExFmt<T>::RB + (((2 * g + hf) ^ ex_swz<T>(c)) << 4));
}

template <typename T>
__device__ __forceinline__ f32x16_t ex_mfma(u32x4_t a, u32x4_t b, f32x16_t acc) {
  if constexpr (ExFmt<T>::ES == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc,
                                                   0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
    return acc;
  }
}

__device__ __forceinline__ f32x16_t ex_zero16() {
  return f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// tile (32 rows x 64) times the rows in `f`: result rows = tile rows, columns = f's rows.
template <typename T>
__device__ __forceinline__ f32x16_t ex_rows_product(const char* tile, const ExRow<T>& f, int c, int hf) {
  f32x16_t acc = ex_zero16();
#pragma unroll
  for (int g = 0; g < ExFmt<T>::NG; ++g) acc = ex_mfma<T>(ex_tile_chunk<T>(tile, c, hf, g), f.v[g], acc);
  return acc;
}

// What rounding a and b to the bfloat16 pair w took off, as such a pair.
__device__ __forceinline__ uint32_t ex_pack_rest(float a, float b, uint32_t w) {
  return pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
}

// y[cc] += tile^T x over the tile's 32 rows: rows of y are columns 32 cc .. 32 cc + 31 of the
// tile. In bf16 x is rounded to bf16 for the product, half a step of the result's own type; FINE: what the
// rounding took off is multiplied too, in products of its own. Calls of few keys or queries take that: a result's
// error in norm is then the 1.66e-3 of its own rounding, instead of 2.3e-3 to 2.4e-3. For long rows it would cost 20
// to 50% (4 x 4096 tokens, 12 heads, forward 204 and 310 us, with the backward pass 924 and 1348; 16 x 512 with a
// bias 120 and 145; 8 x 1057 under a window 96 and 118).
template <typename T, bool FINE = false>
__device__ __forceinline__ void ex_cols_product(f32x16_t (&y)[2], const char* tile, const f32x16_t& x, int lane) {
  const int hf = lane >> 5;
  if constexpr (ExFmt<T>::ES == 2) {
    const int i16 = lane & 15, r0 = 4 * hf + (i16 >> 2);
#pragma unroll
    for (int pp = 0; pp < 2; ++pp) {
      u32x4_t b, t[2];
#pragma unroll
      for (int w = 0; w < 4; ++w) b[w] = pack_bf16x2(x[8 * pp + 2 * w], x[8 * pp + 2 * w + 1]);
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        typedef short v4i16 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
        const int col = 32 * cc + 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
        uint2 h[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int row = 16 * pp + 8 * k + r0;
          const char* at = tile + row * 128 + (((col >> 3) ^ ex_swz<T>(row)) << 4) + (col & 7) * 2;
          h[k] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)at));
        }
        t[cc] = u32x4_t{h[0].x, h[0].y, h[1].x, h[1].y};
        y[cc] = ex_mfma<T>(t[cc], b, y[cc]);
      }
      if constexpr (FINE) {
#pragma unroll
        for (int w = 0; w < 4; ++w) b[w] = ex_pack_rest(x[8 * pp + 2 * w], x[8 * pp + 2 * w + 1], b[w]);
#pragma unroll
        for (int cc = 0; cc < 2; ++cc) y[cc] = ex_mfma<T>(t[cc], b, y[cc]);
      }
    }
  } else {
    const int ln = ex_opaque(lane), h4 = (ln >> 5) * 4;  // 32 addresses, taken anew rather than kept in registers
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = (r & 3) + 8 * (r >> 2) + h4;
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const int col = 32 * cc + (ln & 31);
        const float a =
            *reinterpret_cast<const float*>(tile + row * 256 + (((col >> 2) ^ ex_swz<T>(row)) << 4) + (col & 3) * 4);
        y[cc] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, x[r], y[cc], 0, 0, 0);
      }
    }
  }
}

// ------------------------------------------------------------------ bf16 tiles of 64 rows
// Shared by a block of four waves and loaded by all of them: wave w takes rows 8 w .. 8 w + 7 and
// those 32 further. Offset of a lane's 16 bytes in memory for a row pitch, and the operands.
constexpr int kTile64 = 64 * 128;  // bytes

// COLS: a tile that is read by columns only, with a permutation of period 4.
__device__ __forceinline__ int ex_swz_cols(int r) { return ((r & 1) << 1) | ((r & 2) << 1); }
template <bool COLS = false>
__device__ __forceinline__ uint32_t ex_load64(int wave, int lane, int pitch) {
  const int row = 8 * wave + (lane >> 3);
  return (uint32_t)(row * pitch + (((lane & 7) ^ (COLS ? ex_swz_cols(row) : ex_swz<uint16_t>(row))) << 4));
}
// The tiles of a matrix that a block loads one after another: where the next one begins and how many
// rows there are from there on, in scalar registers (few scalar instructions per tile: where a SIMD
// has one wave, every instruction costs it about five cycles).
struct ExStream {
  const char* at;
  int rows;
};
__device__ __forceinline__ ExStream ex_stream(const char* base, int pitch, int row0, int limit) {
  return ExStream{base + (int64_t)row0 * pitch, limit - row0};
}
__device__ __forceinline__ void ex_load_next64(ExStream& m, int pitch, uint32_t off, uint32_t lds, int wave) {
  const int half = 32 * pitch, bytes = max((min(m.rows, 64) - 1) * pitch + 128, 0);
  auto words = [](const char* p, int n) __attribute__((always_inline)) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    u32x4_t w;
    w[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    w[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(a >> 32) & 0xffffu));
    w[2] = (uint32_t)__builtin_amdgcn_readfirstlane(n);
    w[3] = 0x00020000u;
    return w;
  };
  ex_load_lds16(words(m.at, bytes), off, lds + 1024u * wave);
  ex_load_lds16(words(m.at + half, max(bytes - half, 0)), off, lds + 4096u + 1024u * wave);
  m.at += 2 * (int64_t)half;
  m.rows -= 64;
}

// The lane's byte addresses in a tile: row c, chunks 2 g + hf; and the transposing reads of rows
// 4 hf + (lane % 16) / 4, columns 32 cc ... (rows 8 further: col8, which a COLS tile does not need).
template <bool COLS>
struct ExCols64 {
  int col[2], col8[COLS ? 1 : 2];
};
struct ExRows64 {
  int row[4];
};
__device__ __forceinline__ ExRows64 ex_rows64(int lane) {
  ExRows64 a;
  const int c = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int g = 0; g < 4; ++g) a.row[g] = c * 128 + (((2 * g + hf) ^ ex_swz<uint16_t>(c)) << 4);
  return a;
}
template <bool COLS>
__device__ __forceinline__ ExCols64<COLS> ex_cols64(int lane) {
  ExCols64<COLS> a;
  const int hf = lane >> 5, i16 = lane & 15, row = 4 * hf + (i16 >> 2);
#pragma unroll
  for (int cc = 0; cc < 2; ++cc) {
    const int col = 32 * cc + 16 * ((lane >> 4) & 1) + 4 * (i16 & 3);
    auto at = [&](int r) { return r * 128 + (((col >> 3) ^ (COLS ? ex_swz_cols(r) : ex_swz<uint16_t>(r))) << 4) + (col & 7) * 2; };
    a.col[cc] = at(row);
    if constexpr (!COLS) a.col8[cc] = at(row + 8);
  }
  return a;
}
__device__ __forceinline__ u32x4_t ex_read_row(const char* tile, const ExRows64& a, int half, int g) {
  return *reinterpret_cast<const u32x4_t*>(tile + a.row[g] + half * 4096);
}
// Rows 32 half + 16 pp .. + 15 of columns 32 cc .. as the first operand of a product over rows.
template <bool COLS>
__device__ __forceinline__ u32x4_t ex_read_col(const char* tile, const ExCols64<COLS>& a, int half, int pp, int cc) {
  typedef short v4i16 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
  const int o = half * 4096 + pp * 2048, o8 = COLS ? a.col[cc] + 1024 : a.col8[COLS ? 0 : cc];
  const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(tile + a.col[cc] + o)));
  const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(tile + o8 + o)));
  return u32x4_t{lo.x, lo.y, hi.x, hi.y};
}

// 32 rows of 64 sums, y[cc][r] = column 32 cc + 8 (r / 4) + 4 hf + r % 4 of row c, times `scale`, to
// bf16 rows in memory: through LDS (`st`, 32 x 144 bytes of the wave's own), so that eight lanes
// write a whole row. Rows r >= rows are left out.
__device__ __forceinline__ void ex_store_rows32(char* st, const f32x16_t (&y)[2], float scale, char* out, int64_t pitch,
                                                int rows, int lane) {
  const int c = lane & 31, hf = lane >> 5;
#pragma unroll
  for (int cc = 0; cc < 2; ++cc)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<uint2*>(st + c * 144 + 64 * cc + 16 * (r >> 2) + 8 * hf) =
          make_uint2(pack_bf16x2(y[cc][r] * scale, y[cc][r + 1] * scale), pack_bf16x2(y[cc][r + 2] * scale, y[cc][r + 3] * scale));
  wave_lds_sync();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int row = 8 * k + (lane >> 3);
    const uint4 v = *reinterpret_cast<const uint4*>(st + row * 144 + 16 * (lane & 7));
    if (row < rows) *reinterpret_cast<uint4*>(out + row * pitch + 16 * (lane & 7)) = v;
  }
  wave_lds_sync();
}

// Keeps the computation of x before this point and what follows behind it.
template <typename T>
__device__ __forceinline__ void ex_pin(T& x) { asm volatile("" : "+v"(x)); }

// The rows tile and (batch row, head) `pair` of block `bid`: the tiles of a pair on one XCD where the pairs
// come in eights. `uneven`: every pair's tile 0 before any tile 1, where a mask makes some tiles far
// longer than others, which then start first.
__device__ __forceinline__ void ex_block_pair(int bid, int tiles, int pairs, bool uneven, int& qt, int& pair) {
  if (uneven) {
    qt = bid / pairs;
    pair = bid % pairs;
  } else if (pairs % 8 == 0) {
    const int G = 8 * tiles, w = bid % G;
    pair = bid / G * 8 + w % 8;
    qt = w / 8;
  } else {
    pair = bid / tiles;
    qt = bid % tiles;
  }
}

// ------------------------------------------------------------------ lanes
// The value of the other half's lane (l ^ 32).
__device__ __forceinline__ float ex_other_half(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}
__device__ __forceinline__ float ex_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// ------------------------------------------------------------------ which pairs attend
struct ExRow0 {  // a batch row's lengths and first position
  int qlen, klen, pos;
};
__device__ __forceinline__ ExRow0 ex_batch_row(const ExactParams& p, int b) {
  ExRow0 r;
  r.qlen = p.q_lens ? min(max(p.q_lens[b], 0), p.nq) : p.nq;
  r.klen = p.kv_lens ? min(max(p.kv_lens[b], 0), p.nk) : p.nk;
  r.pos = p.q_pos ? min(max(p.q_pos[b], -(1 << 26)), 1 << 26) : 0;
  return r;
}

// x attends when x - lo <= span (unsigned), or x = extra.
struct ExSpan {
  int lo;
  unsigned span;
  int extra;
};
__device__ __forceinline__ bool ex_in(const ExSpan& s, int x) { return (unsigned)(x - s.lo) <= s.span || x == s.extra; }
// Masks a tile whose first key (or query) of the lane is x0. `one`: the wave knows that no lane's extra one
// is in the tile.
__device__ __forceinline__ void ex_mask(f32x16_t& s, const ExSpan& a, int x0, bool one) {
  const int d = x0 - a.lo;
  if (one) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = (unsigned)(d + (r & 3) + 8 * (r >> 2)) <= a.span ? s[r] : -INFINITY;
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = ex_in(a, x0 + (r & 3) + 8 * (r >> 2)) ? s[r] : -INFINITY;
  }
}
__device__ __forceinline__ ExSpan ex_span(int lo, int hi, int extra) {
  return hi < lo ? ExSpan{0x40000000, 0u, extra} : ExSpan{lo, (unsigned)(hi - lo), extra};
}
// The keys of the query at position pos.
__device__ __forceinline__ ExSpan ex_keys_of(const ExactParams& p, int pos, int klen) {
  int lo = 0, hi = klen - 1, extra = -1;
  if (p.causal) hi = min(hi, pos);
  if (p.window && pos != 0) {
    lo = max(0, pos - p.half);
    hi = min(hi, pos + p.half);
    if (klen > 0 && (!p.causal || pos >= 0)) extra = 0;
  }
  return ex_span(lo, hi, extra);
}
// The query rows of key j.
__device__ __forceinline__ ExSpan ex_queries_of(const ExactParams& p, const ExRow0& r, int j) {
  if (j >= r.klen) return ExSpan{0x40000000, 0u, -1};
  int lo = 0, hi = r.qlen - 1, extra = -1;
  if (p.causal) lo = max(lo, j - r.pos);
  if (p.window && j != 0) {
    lo = max(lo, j - p.half - r.pos);
    hi = min(hi, j + p.half - r.pos);
    if (!p.causal && -r.pos >= 0 && -r.pos < r.qlen) extra = -r.pos;
  }
  return ex_span(lo, hi, extra);
}

// The tiles (of 32 or 64 rows) that a block visits: an extra one first (the global key or query of a
// window), then lo .. hi. `n` of them.
struct ExTiles {
  int first, lo, n;  // first < 0: none
};
__device__ __forceinline__ int ex_tile_at(const ExTiles& t, int i) {
  return t.first >= 0 ? (i == 0 ? t.first : t.lo + i - 1) : t.lo + i;
}
template <int TILE>
__device__ __forceinline__ ExTiles ex_tiles(int lo, int hi, int extra) {  // of elements
  ExTiles t{-1, 0, 0};
  if (hi >= lo) {
    t.lo = lo / TILE;
    t.n = hi / TILE - t.lo + 1;
  }
  if (extra >= 0 && (t.n == 0 || extra / TILE < t.lo || extra / TILE >= t.lo + t.n)) {
    t.first = extra / TILE;
    t.n += 1;
  }
  return t;
}
// Key tiles of the queries at positions pmin .. pmax; `all`: a global query among them counts.
template <int TILE = 32>
__device__ __forceinline__ ExTiles ex_key_tiles(const ExactParams& p, int pmin, int pmax, int klen, bool all = true) {
  int lo = 0, hi = klen - 1, extra = -1;
  if (p.causal) hi = min(hi, pmax);
  if (p.window && (!all || p.causal || pmin > 0 || pmax < 0)) {  // no global query with keys of its own
    lo = max(0, pmin - p.half);
    hi = min(hi, pmax + p.half);
    if (klen > 0 && (!p.causal || pmax >= 0)) extra = 0;
  }
  return ex_tiles<TILE>(lo, hi, extra);
}
// Query tiles of the keys jmin .. jmax (jmax < klen).
template <int TILE = 32>
__device__ __forceinline__ ExTiles ex_query_tiles(const ExactParams& p, const ExRow0& r, int jmin, int jmax) {
  int lo = 0, hi = r.qlen - 1, extra = -1;
  if (jmax < jmin) return ExTiles{-1, 0, 0};
  if (p.causal) lo = max(lo, jmin - r.pos);
  if (p.window && jmin > 0) {
    lo = max(lo, jmin - p.half - r.pos);
    hi = min(hi, jmax + p.half - r.pos);
    if (!p.causal && -r.pos >= 0 && -r.pos < r.qlen) extra = -r.pos;
  }
  return ex_tiles<TILE>(lo, hi, extra);
}
// Under a window the kernels of 128 rows leave the 32 rows around a global row, whose way over the keys (or
// queries) is far longer than the others', to blocks of their own at the grid's beginning, whose four waves
// share it. The first of those 32 query rows, -1 if there is none: causal queries have no such row.
__device__ __forceinline__ int ex_global_rows(const ExactParams& p, const ExRow0& r) {
  return p.window && !p.causal && -r.pos >= 0 && -r.pos < r.qlen ? -r.pos / 32 * 32 : -1;
}
// Where part k of n begins among `all` tiles.
__device__ __forceinline__ int ex_part(int all, int k, int n) { return (int)((int64_t)all * k / n); }
// Whether every query at pmin .. pmax attends every key of k0 .. k0 + 31.
__device__ __forceinline__ bool ex_whole(const ExactParams& p, int pmin, int pmax, int k0, int klen) {
  bool w = k0 + 32 <= klen;
  if (p.causal) w = w && k0 + 31 <= pmin;
  if (p.window) w = w && k0 >= pmax - p.half && k0 + 31 <= pmin + p.half;
  return w;
}

// The same as a range: of first keys k0 for queries at pmin .. pmax, and of first positions q0 of 32 queries
// for the keys j0 .. j0 + 31 (none where those pass klen).
struct ExRange {
  int lo, hi;
};
__device__ __forceinline__ bool ex_has(const ExRange& r, int x) { return x >= r.lo && x <= r.hi; }
__device__ __forceinline__ ExRange ex_whole_keys(const ExactParams& p, int pmin, int pmax, int klen) {
  ExRange r{-0x40000000, klen - 32};
  if (p.causal) r.hi = min(r.hi, pmin - 31);
  if (p.window) r = ExRange{pmax - p.half, min(r.hi, pmin + p.half - 31)};
  return r;
}
__device__ __forceinline__ ExRange ex_whole_queries(const ExactParams& p, int j0, int klen) {
  ExRange r{-0x40000000, j0 + 32 <= klen ? 0x40000000 : -0x40000001};
  if (p.causal) r.lo = j0 + 31;
  if (p.window) r = ExRange{max(r.lo, j0 + 31 - p.half), min(r.hi, j0 + p.half - 31)};
  return r;
}
// Positions of the rows that attend more than one key, as far as lengths, causality and window say. In a row
// outside P is 1 or 0 and dS is zero; its sums would leave their rounding instead, which is all there is of
// a gradient where no row attends more (one token).
__device__ __forceinline__ ExRange ex_many_keys(const ExactParams& p, int klen) {
  if (klen < 2) return ExRange{1, 0};
  ExRange r{p.causal ? 1 : -0x40000000, 0x40000000};
  if (p.window) r = ExRange{max(r.lo, 1 - p.half), klen - 1 + p.half};
  return r;
}
// Zeros dS of such rows in a half tile whose queries begin at position q0.
__device__ __forceinline__ void ex_drop_single(f32x16_t& d, const ExRange& many, int q0, int hf) {
  if (__builtin_expect(q0 < many.lo || q0 + 31 > many.hi, 0)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = ex_has(many, q0 + 4 * hf + (r & 3) + 8 * (r >> 2)) ? d[r] : 0.f;
  }
}

// ------------------------------------------------------------------ relative bias
// Bucket of the key rel = j - p places behind the query: distances below E have one each, distance
// d >= E the bucket E + (number of thresholds <= d); the buckets of rel > 0 follow those of rel <= 0.
__device__ __forceinline__ int ex_bucket(const ExactParams& p, int rel) {
  int d = p.bidirectional ? abs(rel) : max(-rel, 0);
  int n = d;
  if (d >= p.E) {
    n = p.E;
    for (int k = 0; k < p.nthr; ++k) n += p.thr[k] <= d ? 1 : 0;
  }
  return n + (p.bidirectional && rel > 0 ? p.side : 0);
}
template <typename T>
__device__ __forceinline__ float ex_elem(const void* base, int64_t i) {
  return load_f32(static_cast<const T*>(base), i);
}
// Fills heads h0 .. h0 + nh - 1 of a table in LDS: entry rel + D + 64 of a head's 2 D + 129 is the bias
// of rel in base-2 units. A value that masks (-1e30 and below) becomes -inf.
template <typename T>
__device__ __forceinline__ void ex_fill_bias(const ExactParams& p, float* tb, int h0, int nh) {
  const int n = 2 * p.D + 129;
  for (int e = threadIdx.x; e < n; e += blockDim.x) {
    const int c = ex_bucket(p, min(max(e - p.D - 64, -p.D), p.D));
    for (int g = 0; g < nh; ++g) {
      const float v = ex_elem<T>(p.table, (int64_t)c * p.H + h0 + g);
      tb[g * n + e] = v <= -1e30f ? -INFINITY : v * kLog2e;
    }
  }
}
// Where a tile lies: 0 near (its pairs need entries of their own), -1 all rel <= -D, 1 all rel >= D.
__device__ __forceinline__ int ex_bias_side(const ExactParams& p, int k0, int pmin, int pmax) {
  return k0 + 31 - pmin <= -p.D ? -1 : k0 - pmax >= p.D ? 1 : 0;
}

}  // namespace mca
