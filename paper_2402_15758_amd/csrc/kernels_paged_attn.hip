// Attention of new tokens over a paged K/V cache (paged.h): causal, grouped heads,
// optionally a window behind a few first positions that stay visible.
//
// The query heads that share a cache head are rows of one operand: query v of a
// sequence and cache head kvh is row v / group, head kvh group + v % group.
#include <algorithm>

#include "common.h"
#include "paged.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

// ---- which queries, which positions ----------------------------------------------
struct QueryBlock {
  int b, row0, n;           // sequence, its first row, positions before it
  int v0, count;            // first query, queries (0: nothing here)
};
__device__ __forceinline__ int clamp_row(const PagedAttnArgs& a, int r) { return min(max(r, 0), a.rows); }

// Block `slot` of BQ queries.  All lanes of a wave; the result is uniform.
template <int BQ>
__device__ __forceinline__ QueryBlock find_block(const PagedView& c, const PagedAttnArgs& a, int slot) {
  QueryBlock k;
  int rows = 1, at;
  if (a.row0 == nullptr) {
    const int per = (a.group + BQ - 1) / BQ;
    k.b = slot / per;
    k.row0 = k.b;
    at = slot - k.b * per;
  } else {
    // the last sequence whose slots start at or before this one, 64 looked at at once
    const int lane = threadIdx.x & 63;
    int lo = 0, len = c.B;
    bool none = false;
    do {
      const int step = (len + 63) / 64, i = lo + lane * step;
      const bool before =
          lane * step < len && (int)((int64_t)clamp_row(a, a.row0[i]) * a.group / BQ) + i <= slot;
      const int k64 = __popcll(__ballot(before));
      none = none || k64 == 0;
      const int skip = max(k64 - 1, 0) * step;
      lo += skip;
      len = min(step, len - skip);
    } while (len > 1);
    k.b = __builtin_amdgcn_readfirstlane(lo);
    k.row0 = clamp_row(a, a.row0[k.b]);
    rows = none ? 0 : max(clamp_row(a, a.row0[k.b + 1]) - k.row0, 0);
    at = slot - ((int)((int64_t)k.row0 * a.group / BQ) + k.b);
  }
  k.v0 = at * BQ;
  k.count = max(min(rows * a.group - k.v0, BQ), 0);
  k.n = min(a.n_b[k.b], 1 << 30);
  return k;
}

// The tiles of TILE positions that some query of a block sees: `lead` ones from
// position 0 (the first positions that stay visible), then those from tile `first`.
template <int TILE>
struct Span {
  int p_lo, p_hi;           // first and last query's position
  int lead, first, tiles;
  __device__ __forceinline__ Span(const PagedView& c, const PagedAttnArgs& a, const QueryBlock& k) {
    p_lo = k.n + k.v0 / a.group;
    p_hi = k.n + (k.v0 + max(k.count, 1) - 1) / a.group;
    const int last = min(p_hi, c.cap - 1);
    const int from = a.window > 0 ? max(p_lo - a.window + 1, 0) : 0;
    first = from / TILE;
    lead = a.window > 0 ? min((min(a.sinks, from) + TILE - 1) / TILE, first) : 0;
    // a cache shorter than the first positions
    lead = min(lead, (c.cap + TILE - 1) / TILE);
    tiles = k.n < 0 || k.count == 0 ? 0 : lead + max(last / TILE - first + 1, 0);
  }
  __device__ __forceinline__ int tile(int t) const { return t < lead ? t : first + (t - lead); }
};
// Parts that a block's tiles are dealt in.
__device__ __forceinline__ int parts_of(int tiles, int splits, int least) {
  return max(min(splits, (tiles + least - 1) / least), 1);
}

// The low n bits (none below 1, all from 32 on).
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
// Positions base .. base + 31 that the query at position p sees.
__device__ __forceinline__ uint32_t seen_bits(const PagedAttnArgs& a, int base, int p) {
  const uint32_t causal = low_bits(p + 1 - base);
  return a.window == 0 ? causal : causal & (~low_bits(p + 1 - a.window - base) | low_bits(a.sinks - base));
}
// Those that some query at a position p_lo .. p_hi sees, and that all of them see.
__device__ __forceinline__ bool some_see(const PagedAttnArgs& a, int pos, int p_lo, int p_hi) {
  return pos <= p_hi && (a.window == 0 || pos > p_lo - a.window || pos < a.sinks);
}
__device__ __forceinline__ bool all_see(const PagedAttnArgs& a, int from, int to, int p_lo, int p_hi) {
  return to <= p_lo && (a.window == 0 || from > p_hi - a.window || to < a.sinks);
}

// ---- softmax state ---------------------------------------------------------------
// m: the running maximum of scale2 s, -inf where nothing was seen, and no less than
// UNKNOWN where something was: a scaled score past the float's range weighs nothing
// if negative and makes the row NaN if positive, and a row of nothing but negative
// ones is 0 / 0.
constexpr float UNKNOWN = -__FLT_MAX__;
// A weight enters the bf16 MFMA rounded once, 2^-9 of itself on average as much as the
// result's own rounding adds.  More terms would halve what weights of mixed roundings
// leave, and make a visible infinity of V NaN (its product with the second term).
__device__ __forceinline__ float weight(float a, float b) {  // 2^(a - b), 0 from nothing
  return a == -CH_INF ? 0.f : __builtin_amdgcn_exp2f(a - b);
}
__device__ __forceinline__ uint32_t cvt_pk_bf16(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}
template <typename T>
__device__ __forceinline__ bool any_nonfinite(int4 v);
template <>
__device__ __forceinline__ bool any_nonfinite<bf16_t>(int4 v) {
  auto bad = [](int w) { return (w & 0x7f80) == 0x7f80 || (w & 0x7f800000) == 0x7f800000; };
  return bad(v.x) || bad(v.y) || bad(v.z) || bad(v.w);
}
template <>
__device__ __forceinline__ bool any_nonfinite<float>(int4 v) {
  auto bad = [](int w) { return (w & 0x7f800000) == 0x7f800000; };
  return bad(v.x) || bad(v.y) || bad(v.z) || bad(v.w);
}

// DV values of one row into the caller's output.
template <typename T, int DV>
__device__ __forceinline__ void store_out(T* p, const float* x, bool vec) {
  if (!vec) {
#pragma unroll
    for (int i = 0; i < DV; ++i) p[i] = ET<T>::from_f(x[i]);
  } else if constexpr (sizeof(T) == 2) {
    uint32_t w[DV / 2];
#pragma unroll
    for (int i = 0; i < DV / 2; ++i) w[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
    if constexpr (DV == 8)
      st16(p, int4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]});
    else
      *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
  } else {
#pragma unroll
    for (int i = 0; i < DV; i += 4) *reinterpret_cast<float4*>(p + i) = float4{x[i], x[i + 1], x[i + 2], x[i + 3]};
  }
}

// ---- few queries -----------------------------------------------------------------
// A workgroup takes 16 queries of one cache head and a part of their positions, its
// four waves every fourth tile of 32 positions, and joins the waves' states in LDS.
//
// S^T = K Q^T: 16x16 MFMAs, a lane 16 bytes of a key's row a step.  Lane (g, c16)
// then holds query c16 and keys 16 t + 4 g + r, which is the operand layout of P^T
// for O^T += V^T P^T with the keys of a block of 32 in that order: P stays in
// registers.  V^T needs eight keys of one dimension in a lane; lane (g, c16) loads
// HD / 16 dimensions of exactly its group's keys, whole rows by 16 lanes, and pairs
// them by byte permutes, so V needs no LDS either.  O^T's row 4 g + r of MFMA j is
// dimension (4 g + r) HD / 16 + j.
template <typename T, int HD>
struct RowTile {
  static constexpr int VEC = ET<T>::VEC, KB = 4 * VEC, KS = HD / KB;
  static constexpr int DV = HD / 16;                    // dimensions of a lane
  static constexpr int VW = DV * (int)sizeof(T) / 4;    // their words
  int4 k[2][KS];
  uint32_t v[8][VW];
};

template <typename T, int HD>
__device__ __forceinline__ void load_v(uint32_t* w, const T* p) {
  constexpr int VW = RowTile<T, HD>::VW;
  if constexpr (VW == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x, w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < VW; i += 4) {
      const int4 x = ld16(p + i * 4 / (int)sizeof(T));
      w[i] = x.x, w[i + 1] = x.y, w[i + 2] = x.z, w[i + 3] = x.w;
    }
  }
}

// O^T += V^T P^T over 32 keys.  p: the weights packed as the bf16 operand; f32 takes s
// itself.
template <typename T, int HD>
__device__ __forceinline__ void row_pv(const uint32_t (&v)[8][RowTile<T, HD>::VW], const f32x4 (&s)[2], int4 p,
                                       f32x4 (&o)[HD / 16]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int m = 0; m < 4; ++m)
        w[m] = __builtin_amdgcn_perm(v[2 * m + 1][j / 2], v[2 * m][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
      const int4 vf = int4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
      o[j] = mfma_kb<T>(vf, p, o[j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < HD / 16; ++j)
        o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][j]), s[i / 4][i % 4], o[j], 0, 0, 0);
  }
}

constexpr int RB = 16, RT = 32;  // queries and positions of a wave's tile
constexpr int R_LEAST = 8;       // tiles of a part: two a wave

template <typename T, int HD>
__global__ __launch_bounds__(256) void paged_rows_kernel(const PagedView c, const PagedAttnArgs a) {
  typedef RowTile<T, HD> Tile;
  constexpr int DV = Tile::DV, KS = Tile::KS;
  __shared__ float osh[4][RB][HD + 4];
  __shared__ float msh[4][RB], lsh[4][RB];
  const int kvh = blockIdx.x % c.H, rest = blockIdx.x / c.H;
  const int split = rest % a.splits, slot = rest / a.splits;
  const QueryBlock blk = find_block<RB>(c, a, slot);
  if (blk.count == 0) return;
  const Span<RT> span(c, a, blk);
  const int parts = parts_of(span.tiles, a.splits, R_LEAST);
  if (split >= parts) return;
  const int t0 = (int)((int64_t)span.tiles * split / parts), t1 = (int)((int64_t)span.tiles * (split + 1) / parts);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int* ptab = c.page_table + (int64_t)blk.b * c.max_pages;
  const T* pool = (const T*)c.pool;

  const int vq = blk.v0 + min(c16, blk.count - 1);
  const int qrow = vq / a.group;
  const int qpos = blk.n + qrow;
  int4 qf[KS];
  {
    const int flip = a.flip == 0 ? 0 : (sizeof(T) == 2 ? (int)0x80008000 : (int)0x80000000);
    const T* q = (const T*)a.q + (int64_t)(blk.row0 + qrow) * a.ldq + (kvh * a.group + vq - qrow * a.group) * HD;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int4 x = ld16(q + ks * Tile::KB + g * Tile::VEC);
      qf[ks] = int4{x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip};
    }
  }
  float m = -CH_INF, l = 0.f;
  f32x4 o[DV];
#pragma unroll
  for (int j = 0; j < DV; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int t = t0 + wave; t < t1; t += 4) {
    const int base = span.tile(t) * RT;
    const int pos = base + (lane & 31);
    // a row that no query sees is read as row 0 of the pool and counts for nothing
    const uint32_t row = some_see(a, pos, span.p_lo, span.p_hi) ? paged_row(c, ptab, pos) : PAGED_NONE;
    const uint32_t held = (uint32_t)__ballot(row != PAGED_NONE);
    const int safe = row == PAGED_NONE ? 0 : (int)row;
    Tile x;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t r = (uint32_t)__shfl(safe, 16 * h + c16) + (uint32_t)(kvh * c.ps.d);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x.k[h][ks] = ld16(pool + (uint64_t)r * HD + ks * Tile::KB + g * Tile::VEC);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t r = (uint32_t)__shfl(safe, 16 * (i / 4) + 4 * g + i % 4) + (uint32_t)((c.H + kvh) * c.ps.d);
      load_v<T, HD>(x.v[i], pool + (uint64_t)r * HD + c16 * DV);
    }
    f32x4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[h] = mfma_kb<T>(x.k[h][ks], qf[ks], s[h]);
    }
    const bool whole = held == ~0u && all_see(a, base, base + RT - 1, span.p_lo, span.p_hi);
    const uint32_t vis = whole ? ~0u : held & seen_bits(a, base, qpos);
    const uint32_t mine = vis >> (4 * g);
    float mx = -CH_INF;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, (mine >> (16 * h + r)) & 1 ? s[h][r] : -CH_INF);
    mx = rows_max(mx);
    const float mn = vis != 0 ? fmaxf(m, fmaxf(mx * a.scale2, UNKNOWN)) : m;
    const float al = m == mn ? 1.f : weight(m, mn);
    m = mn;
    float ls = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[h][r], a.scale2, -mn));
        s[h][r] = (mine >> (16 * h + r)) & 1 ? p : 0.f;
        ls = ls + s[h][r];
      }
    l = fmaf(l, al, ls);
    if (__ballot(al != 1.f) != 0) {
#pragma unroll
      for (int j = 0; j < DV; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][r] = o[j][r] * al;
    }
    int4 pf = {};
    if constexpr (sizeof(T) == 2)
      pf = int4{(int)cvt_pk_bf16(s[0][0], s[0][1]), (int)cvt_pk_bf16(s[0][2], s[0][3]),
                (int)cvt_pk_bf16(s[1][0], s[1][1]), (int)cvt_pk_bf16(s[1][2], s[1][3])};
    if (whole) {
      row_pv<T, HD>(x.v, s, pf, o);
      continue;
    }
    // A masked tile: values of rows that no query sees are zeros, and an infinity or a
    // NaN in a row that some queries see and others do not must not reach the others
    // through 0 x inf.  Where there is one, the tile is multiplied a query at a time.
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool on = (held >> (16 * (i / 4) + 4 * g + i % 4)) & 1;
#pragma unroll
      for (int w = 0; w < Tile::VW; ++w) x.v[i][w] = on ? x.v[i][w] : 0u;
#pragma unroll
      for (int w = 0; w < Tile::VW; w += 2)
        odd = odd || any_nonfinite<T>(int4{(int)x.v[i][w], (int)x.v[i][w + 1], 0, 0});
    }
    if (__ballot(odd) == 0) {
      row_pv<T, HD>(x.v, s, pf, o);
    } else {
      for (int q = 0; q < RB; ++q) {
        const uint32_t vq_bits = (uint32_t)__builtin_amdgcn_readlane((int)vis, q);
        uint32_t v[8][Tile::VW];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int w = 0; w < Tile::VW; ++w)
            v[i][w] = (vq_bits >> (16 * (i / 4) + 4 * g + i % 4)) & 1 ? x.v[i][w] : 0u;
        f32x4 oq[DV];
#pragma unroll
        for (int j = 0; j < DV; ++j) oq[j] = o[j];
        row_pv<T, HD>(v, s, pf, oq);
#pragma unroll
        for (int j = 0; j < DV; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[j][r] = c16 == q ? oq[j][r] : o[j][r];
      }
    }
  }
  l = rows_sum(l);
  // the four waves' states, joined in wave order
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < DV; ++j) osh[wave][c16][(4 * g + r) * DV + j] = o[j][r];
  if (g == 0) msh[wave][c16] = m, lsh[wave][c16] = l;
  __syncthreads();
  const int q = tid / 16, d0 = (tid % 16) * DV;
  float mt = msh[0][q];
#pragma unroll
  for (int w = 1; w < 4; ++w) mt = fmaxf(mt, msh[w][q]);
  float lt = 0.f, x[DV];
#pragma unroll
  for (int j = 0; j < DV; ++j) x[j] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (msh[w][q] == -CH_INF) continue;  // that wave saw nothing
    const float f = __builtin_amdgcn_exp2f(msh[w][q] - mt);
    lt = fmaf(lsh[w][q], f, lt);
#pragma unroll
    for (int j = 0; j < DV; ++j) x[j] = fmaf(osh[w][q][d0 + j], f, x[j]);
  }
  if (q >= blk.count) return;
  if (parts == 1) {
    const int r = (blk.v0 + q) / a.group, h = blk.v0 + q - r * a.group;
#pragma unroll
    for (int j = 0; j < DV; ++j) x[j] = mt == -CH_INF ? 0.f : x[j] / lt;
    store_out<T, DV>((T*)a.out + (int64_t)(blk.row0 + r) * a.ldo + (kvh * a.group + h) * HD + d0, x, a.vec_out != 0);
    return;
  }
  const int64_t at = (((int64_t)slot * c.H + kvh) * a.splits + split) * RB + q;
#pragma unroll
  for (int j = 0; j < DV; j += 4)
    *reinterpret_cast<float4*>(a.part_o + at * HD + d0 + j) = float4{x[j], x[j + 1], x[j + 2], x[j + 3]};
  if (tid % 16 == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = float2{mt, lt};
}

// The parts of a query, joined in order: a wave a query, 64 parts' factors at once.
template <typename T, int HD, int BQ, int TILE>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedView c, const PagedAttnArgs a, int least) {
  const int q0 = blockIdx.x * 4 + (threadIdx.x >> 6);  // query of a slot and cache head
  const int q = q0 % BQ, kvh = q0 / BQ % c.H, slot = q0 / BQ / c.H;
  const int lane = threadIdx.x & 63;
  const QueryBlock blk = find_block<BQ>(c, a, slot);
  if (q >= blk.count) return;
  const Span<TILE> span(c, a, blk);
  const int parts = parts_of(span.tiles, a.splits, least);
  if (parts == 1) return;  // written whole
  const int64_t first = ((int64_t)slot * c.H + kvh) * a.splits * BQ + q;
  float mt = -CH_INF;
  for (int i = lane; i < parts; i += 64) mt = fmaxf(mt, a.part_ml[(first + (int64_t)i * BQ) * 2]);
  mt = wave_max(mt);
  constexpr int D = HD / 64;
  float lt = 0.f, x[D];
#pragma unroll
  for (int j = 0; j < D; ++j) x[j] = 0.f;
  for (int i0 = 0; i0 < parts; i0 += 64) {
    float f = 0.f, fl = 0.f;
    if (i0 + lane < parts) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (first + (int64_t)(i0 + lane) * BQ) * 2);
      f = weight(ml.x, mt);
      fl = f == 0.f && ml.x == -CH_INF ? 0.f : ml.y * f;
    }
    lt = lt + wave_sum(fl);
    const int n = min(64, parts - i0);
    for (int i = 0; i < n; ++i) {
      const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i));
      const float* p = a.part_o + (first + (int64_t)(i0 + i) * BQ) * HD + lane * D;
#pragma unroll
      for (int j = 0; j < D; ++j) x[j] = fmaf(p[j], fi, x[j]);
    }
  }
  const int r = (blk.v0 + q) / a.group, h = blk.v0 + q - r * a.group;
  T* dst = (T*)a.out + (int64_t)(blk.row0 + r) * a.ldo + (kvh * a.group + h) * HD + lane * D;
#pragma unroll
  for (int j = 0; j < D; ++j) dst[j] = ET<T>::from_f(mt == -CH_INF ? 0.f : x[j] / lt);
}

// ---- deal ------------------------------------------------------------------------
constexpr int R_WGS = 1024;  // workgroups that fill the card, four a CU

int64_t row_splits(int64_t cap, int64_t blocks) {
  const int64_t tiles = (cap + RT - 1) / RT + 2;  // a window's ends cut two more
  return std::max<int64_t>(1, std::min((R_WGS + blocks - 1) / blocks, (tiles + R_LEAST - 1) / R_LEAST));
}

template <typename T, int HD>
void attn_go(const PagedView& c, PagedAttnArgs a, void* ws, hipStream_t st) {
  const int64_t slots = paged_attn_slots(a.row0 == nullptr, a.rows, c.B, a.group, RB);
  const int64_t splits = row_splits(c.cap, slots * c.H);
  a.slots = (int)slots;
  a.splits = (int)splits;
  a.part_o = (float*)ws;
  a.part_ml = a.part_o + slots * c.H * splits * RB * HD;
  hipLaunchKernelGGL((paged_rows_kernel<T, HD>), dim3((unsigned)(slots * splits * c.H)), dim3(256), 0, st, c, a);
  if (splits > 1)
    hipLaunchKernelGGL((paged_join_kernel<T, HD, RB, RT>), dim3((unsigned)(slots * c.H * RB / 4)), dim3(256), 0, st, c, a,
                       R_LEAST);
}

}  // namespace

int64_t paged_attn_slots(bool single, int64_t rows, int batch, int group, int block) {
  return single ? (int64_t)batch * ((group + block - 1) / block) : rows * group / block + batch;
}

// Splitting stops where the blocks fill the card, so the partials of any call of up
// to `rows` rows, at most the blocks it has and less than one more round, fit in this.
int64_t paged_attn_bytes(int64_t cap, int rows, int batch, int group, int H, int hd) {
  const int64_t per = (int64_t)RB * (hd + 2) * 4;
  const int64_t blocks = std::max(paged_attn_slots(false, rows, batch, group, RB), paged_attn_slots(true, rows, batch, group, RB)) * H;
  const int64_t most = ((cap + RT - 1) / RT + 2 + R_LEAST - 1) / R_LEAST;
  return std::min(std::min<int64_t>(blocks, R_WGS) * most, (int64_t)2 * R_WGS) * per;
}

void launch_paged_attn(int dtype, const PagedView& c, PagedAttnArgs a, void* ws, hipStream_t st) {
  if (dtype == DT_BF16) {
    if (c.hd == 128)
      attn_go<bf16_t, 128>(c, a, ws, st);
    else
      attn_go<bf16_t, 64>(c, a, ws, st);
  } else if (c.hd == 128) {
    attn_go<float, 128>(c, a, ws, st);
  } else {
    attn_go<float, 64>(c, a, ws, st);
  }
}
