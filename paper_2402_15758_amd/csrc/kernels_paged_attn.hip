// Attention of new tokens over a paged K/V cache (paged.h): causal, grouped heads,
// optionally a window behind a few first positions that stay visible.
//
// The query heads that share a cache head are rows of one operand: query v of a
// sequence and cache head kvh is row v / group, head kvh group + v % group.
#include <algorithm>

#include "common.h"
#include "paged.h"

namespace {

// ---- which queries, which positions ----------------------------------------------
struct QueryBlock {
  int b, row0, n;           // sequence, its first row, positions before it
  int v0, count;            // first query, queries (0: nothing here)
};
__device__ __forceinline__ int clamp_row(const PagedAttnArgs& a, int r) { return min(max(r, 0), a.rows); }

// Block `slot` of BQ queries.  All lanes of a wave; the result is uniform.
//  - a.per > 0: the same number of slots a sequence;
//  - else sequence b's slots start at floor(row0[b] group / BQ) + b, which leaves each
//    room for its own.
template <int BQ>
__device__ __forceinline__ QueryBlock find_block(const PagedView& c, const PagedAttnArgs& a, int slot) {
  QueryBlock k;
  int rows = 1, at;
  if (a.per > 0) {
    k.b = slot / a.per;
    at = slot - k.b * a.per;
    k.row0 = k.b;
    k.n = a.n_b[k.b];
    if (a.row0 != nullptr) {
      k.row0 = clamp_row(a, a.row0[k.b]);
      rows = max(clamp_row(a, a.row0[k.b + 1]) - k.row0, 0);
    }
  } else {
    // the last sequence whose slots start at or before this one, 64 looked at at once;
    // the last look brings all that is needed of it
    const int lane = threadIdx.x & 63;
    int lo = 0, len = c.B;
    for (;;) {
      const int step = (len + 63) / 64, i = lo + min(lane * step, len - 1);
      const int r = clamp_row(a, a.row0[i]);
      const int start = (int)((int64_t)r * a.group / BQ) + i;
      const int last = max(__popcll(__ballot(lane * step < len && start <= slot)) - 1, 0);
      if (step == 1) {
        const int end = clamp_row(a, a.row0[i + 1]), n = a.n_b[i];
        k.b = lo + last;
        k.row0 = __builtin_amdgcn_readlane(r, last);
        k.n = __builtin_amdgcn_readlane(n, last);
        rows = max(__builtin_amdgcn_readlane(end, last) - k.row0, 0);
        at = slot - __builtin_amdgcn_readlane(start, last);
        break;
      }
      lo += last * step;
      len = min(step, len - last * step);
    }
  }
  k.n = max(min(k.n, 1 << 30), -1);
  k.v0 = at * BQ;
  k.count = at < 0 ? 0 : max(min(rows * a.group - k.v0, BQ), 0);
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
// A word's sign bits come out set where an exponent is all ones.
template <typename T>
__device__ __forceinline__ uint32_t odd_bits(uint32_t w) {
  constexpr uint32_t E = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, ONE = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
  return ((w & E) + ONE) & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u);
}

template <typename T, int HD>
__device__ __forceinline__ uint32_t odd_row(const T* p) {
  uint32_t odd = 0;
  for (int i = 0; i < HD; i += 16 / (int)sizeof(T)) {
    const int4 x = ld16(p + i);
    odd |= odd_bits<T>(x.x) | odd_bits<T>(x.y) | odd_bits<T>(x.z) | odd_bits<T>(x.w);
  }
  return odd;
}
// Whether a tile of V in LDS holds an infinity or a NaN; a wave.
template <typename T, int BYTES>
__device__ __forceinline__ bool odd_tile(const char* v, int lane) {
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < BYTES; i += 1024) {
    const int4 x = ld16(v + i + lane * 16);
    odd |= odd_bits<T>(x.x) | odd_bits<T>(x.y) | odd_bits<T>(x.z) | odd_bits<T>(x.w);
  }
  return __ballot(odd != 0) != 0;
}

// A wave's LDS writes before its later reads, by other lanes too.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// A tile that some queries see in part and whose V holds an infinity or a NaN: what a
// query does not see must not reach it, and 0 x inf would carry it through a matrix
// product.  The kernels leave such tiles out and a wave takes them by itself at the
// end, a query at a time over the keys it sees: lanes are keys for the scores and
// dimensions for the sums.  Its queries' states lie in LDS: m, l and o, rows `ldo` apart.
template <typename T, int HD>
__device__ __forceinline__ void tile_alone(const PagedView& c, const PagedAttnArgs& a, const int* ptab, int base, int keys,
                                        const QueryBlock& blk, int v0, int count, int kvh, float* m, float* l,
                                           float* o, int ldo) {
  const int lane = threadIdx.x & 63;
  const T* pool = (const T*)c.pool;
  const int n = blk.n, b_row0 = blk.row0, pos = base + lane;
  const uint32_t row = lane < keys ? paged_row(c, ptab, pos) : PAGED_NONE;
  const uint32_t at = row + (uint32_t)(kvh * c.ps.d);
  constexpr int D = HD / 64;
  for (int i = 0; i < count; ++i) {
    const int qrow = (v0 + i) / a.group, head = kvh * a.group + v0 + i - qrow * a.group;
    bool seen = row != PAGED_NONE && pos <= n + qrow;
    if (a.window > 0) seen = seen && (pos > n + qrow - a.window || pos < a.sinks);
    const uint64_t vis = __ballot(seen);
    if (vis == 0) continue;
    float s = -CH_INF;
    if (seen) {
      const T* q = (const T*)a.q + (int64_t)(b_row0 + qrow) * a.ldq + head * HD;
      const T* k = pool + (uint64_t)at * HD;
      s = 0.f;
      for (int d = 0; d < HD; ++d) s = fmaf(ET<T>::to_f(q[d]), ET<T>::to_f(k[d]), s);
      s = a.flip != 0 ? -s : s;
    }
    const float mn = fmaxf(m[i], fmaxf(wave_max(s) * a.scale2, UNKNOWN));
    const float al = m[i] == mn ? 1.f : weight(m[i], mn);
    float p = seen ? __builtin_amdgcn_exp2f(fmaf(s, a.scale2, -mn)) : 0.f;
    const float ls = wave_sum(p);
    p = ET<T>::to_f(ET<T>::from_f(p));
    float x[D];
#pragma unroll
    for (int d = 0; d < D; ++d) x[d] = o[i * ldo + lane * D + d] * al;
    for (uint64_t rest = vis; rest != 0; rest &= rest - 1) {
      const int key = __ffsll((long long)rest) - 1;
      const float pk = __shfl(p, key);
      const T* vr = pool + (uint64_t)((uint32_t)__shfl((int)at, key) + (uint32_t)(c.H * c.ps.d)) * HD + lane * D;
#pragma unroll
      for (int d = 0; d < D; ++d) x[d] = fmaf(pk, ET<T>::to_f(vr[d]), x[d]);
    }
#pragma unroll
    for (int d = 0; d < D; ++d) o[i * ldo + lane * D + d] = x[d];
    if (lane == 0) {
      l[i] = fmaf(l[i], al, ls);
      m[i] = mn;
    }
    wave_order();
  }
}

// DV values of one row into the caller's output, at any element.
template <typename T, int DV>
__device__ __forceinline__ void store_out(T* p, const float* x) {
  if constexpr (sizeof(T) == 2) {
    typedef uint32_t words __attribute__((ext_vector_type(DV / 2), aligned(2)));
    words w;
#pragma unroll
    for (int i = 0; i < DV / 2; ++i) w[i] = cvt_pk_bf16(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<words*>(p) = w;
  } else {
    typedef float four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int i = 0; i < DV; i += 4) *reinterpret_cast<four*>(p + i) = four{x[i], x[i + 1], x[i + 2], x[i + 3]};
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
//
// Bound by the cache's bytes where few queries read much of it: eight single tokens behind
// 1024 to 4096 positions of 32 heads of 128 (336 MB) 65 us, 5.2 TB/s (69 with each page asked
// for when its tile's turn comes); one behind 32768 of 8 heads (134 MB) 27 us, 5.0 TB/s.
// A wave keeps a tile's K and V in registers, so waves wait for memory by themselves and
// not for each other.
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
  const int parts = parts_of(span.tiles, a.splits, a.least);
  if (split >= parts) return;
  const int t0 = (int)((int64_t)span.tiles * split / parts), t1 = (int)((int64_t)span.tiles * (split + 1) / parts);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int* ptab = c.page_table + (int64_t)blk.b * c.max_pages;
  const T* pool = (const T*)c.pool;

  // The page of a position that some query sees is asked for a tile ahead; a row that none
  // sees is read as row 0 of the pool and counts for nothing.
  int page = 0, slot_in = 0;
  bool seen = false;
  auto ask = [&](int t) {
    const int pos = span.tile(t) * RT + (lane & 31);
    seen = some_see(a, pos, span.p_lo, span.p_hi) && pos < c.cap;
    const int p = seen ? pos : 0, pi = c.ps.quot(p);
    slot_in = p - pi * c.ps.d;
    page = ptab[pi];
  };
  if (t0 + wave < t1) ask(t0 + wave);
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

  bool odd = false;
  for (int t = t0 + wave; t < t1; t += 4) {
    const int base = span.tile(t) * RT;
    const bool there = seen && page >= 0 && page < c.n_pages;
    const uint32_t held = (uint32_t)__ballot(there);
    const int safe = there ? (int)((uint32_t)page * c.page_rows + (uint32_t)slot_in) : 0;
    if (t + 4 < t1) ask(t + 4);
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
    const bool whole = held == ~0u && all_see(a, base, base + RT - 1, span.p_lo, span.p_hi);
    if (!whole) {
      // values of rows that no query sees are zeros
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool on = (held >> (16 * (i / 4) + 4 * g + i % 4)) & 1;
#pragma unroll
        for (int w = 0; w < Tile::VW; ++w) {
          x.v[i][w] = on ? x.v[i][w] : 0u;
          any |= odd_bits<T>(x.v[i][w]);
        }
      }
      if (__ballot(any != 0) != 0) {
        odd = true;
        continue;
      }
    }
    f32x4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[h] = mfma_kb<T>(x.k[h][ks], qf[ks], s[h]);
    }
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
    row_pv<T, HD>(x.v, s, pf, o);
  }
  l = rows_sum(l);
  // the four waves' states, joined in wave order
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < DV; ++j) osh[wave][c16][(4 * g + r) * DV + j] = o[j][r];
  if (g == 0) msh[wave][c16] = m, lsh[wave][c16] = l;
  if (odd) {
    wave_order();
    for (int t = t0 + wave; t < t1; t += 4) {
      const int base = span.tile(t) * RT, pos = base + (lane & 31);
      const uint32_t row = some_see(a, pos, span.p_lo, span.p_hi) ? paged_row(c, ptab, pos) : PAGED_NONE;
      const uint32_t held = (uint32_t)__ballot(row != PAGED_NONE);
      if (held == ~0u && all_see(a, base, base + RT - 1, span.p_lo, span.p_hi)) continue;
      uint32_t any = 0;
      if (row != PAGED_NONE)
        any = odd_row<T, HD>(pool + (uint64_t)(row + (uint32_t)((c.H + kvh) * c.ps.d)) * HD);
      if (__ballot(any != 0) != 0)
        tile_alone<T, HD>(c, a, ptab, base, RT, blk, blk.v0, blk.count, kvh, msh[wave], lsh[wave], &osh[wave][0][0],
                          HD + 4);
    }
  }
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
    store_out<T, DV>((T*)a.out + (int64_t)(blk.row0 + r) * a.ldo + (kvh * a.group + h) * HD + d0, x);
    return;
  }
  const int64_t at = (((int64_t)slot * c.H + kvh) * a.splits + split) * RB + q;
#pragma unroll
  for (int j = 0; j < DV; j += 4)
    *reinterpret_cast<float4*>(a.part_o + at * HD + d0 + j) = float4{x[j], x[j + 1], x[j + 2], x[j + 3]};
  if (tid % 16 == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = float2{mt, lt};
}

// ---- many queries ----------------------------------------------------------------
// A workgroup takes 128 queries of one cache head and a part of their positions, a
// wave 32 of them; tiles of K and V pass through LDS in two buffers, straight from
// memory, the next one on its way while one is used.
//
// S^T = K Q^T by 32x32 MFMAs: a lane holds one query's scores (lane & 31) for half the
// keys, so maxima and sums are one lane's own but for one exchange, and the scores of
// 16 keys are as they stand the operand P^T of O^T += V^T P^T.  16-bit V^T comes from
// LDS's transposed read: within each 16-lane group, lane i receives element i mod 4 of
// the 8-byte blocks addressed by lanes i / 4 + 4 e.  f32 V is read along the row: an
// MFMA's rows are every (HD / 32)th dimension.
//
// A row's 16-byte chunk x lies in place x ^ swizzle(row): the 16 rows of a K read and
// the four rows x 64 bytes of half a transposed read then cover all banks once.
//
// Bound by the chain of scores, exponentials and products, two waves a SIMD: 2048 queries
// of 32 heads of 128 behind 2048 positions take 124 us, 830 TFLOP/s (MFMA busy 34% of the
// time, VALU 38%), behind 14336 positions 525 us, 981; heads of 64 76 us, 680.  32-bit, 2048
// queries of 16 heads behind none: 182 us, 94 of 154 TFLOP/s.  A workgroup of eight waves,
// four buffers with one workgroup a CU, and the next tile's scores beside this tile's
// values took longer or spilt.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int TB = 128;         // queries of a workgroup
template <typename T>
constexpr int TT = sizeof(T) == 2 ? 64 : 32;  // positions of a tile

template <int CH>  // chunks of a row
__device__ __forceinline__ int swizzle(int row) {
  return CH == 8 ? ((row >> 1) & 1) * 4 + ((row >> 2) & 3) : (row & 3) * 4 + ((row >> 2) & 3);
}
__device__ __forceinline__ int2 ld_tr16(const char* p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
  return __builtin_bit_cast(int2, v);
}
__device__ __forceinline__ void dma16(const char* src, char* lds) {  // 16 bytes a lane, 1 KiB a wave
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
// Every load into LDS has landed, every LDS read has its data, on all waves.
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0070);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ uint64_t low_bits64(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

template <typename T, int HD>
struct ManyState {
  static constexpr int KB = TT<T> / 32, ND = HD / 32, QR = HD * (int)sizeof(T) / 32;
  int4 q[QR];            // this lane's query: 16 bytes of every 32
  f32x16 o[ND];
  float m, l;
};

// Where a lane reads in a tile: a key's row for S (its 16-byte piece i at place ^ 32 i),
// its place in V^T's operands.  The steps over pieces, dimension blocks and keys only
// flip chunk bits or add whole rows, so they cost an exclusive or and an immediate.
template <typename T, int HD>
struct LanePlaces {
  static constexpr int ROW = HD * (int)sizeof(T), CH = ROW / 16;
  int k, v;
  __device__ __forceinline__ explicit LanePlaces(int lane) {
    const int c32 = lane & 31, h = lane >> 5;
    k = c32 * ROW + ((h ^ swizzle<CH>(c32)) << 4);
    if constexpr (sizeof(T) == 2) {
      const int g1 = (lane >> 4) & 1, a = lane & 15, key = 4 * h + (a >> 2);
      v = key * ROW + (((2 * g1 + ((a & 3) >> 1)) ^ swizzle<CH>(key)) << 4) + ((a & 1) << 3);
    } else {
      const int at = c32 * (HD / 32) * 4;
      v = 4 * h * ROW + (((at >> 4) ^ h) << 4) + (at & 15);
    }
  }
  __device__ __forceinline__ int key(int kb, int i) const { return (k ^ (32 * i)) + 32 * kb * ROW; }
  // bf16: keys 16 n + 8 e + 4 h .. + 3 of dimension block db
  __device__ __forceinline__ int val16(int n, int e, int db) const {
    return (v ^ (db << 6) ^ (e << 5)) + (16 * n + 8 * e) * ROW;
  }
  // f32: key 8 n + 4 h + j
  __device__ __forceinline__ int val32(int n, int j) const { return (v ^ (j << 6) ^ ((n & 1) << 5)) + (8 * n + j) * ROW; }
  // the sums are cheaper than the registers that would hold them through the loop
  __device__ __forceinline__ void renew() { asm volatile("" : "+v"(k), "+v"(v)); }
};

// V^T's operand of 16 keys.
template <int HD>
__device__ __forceinline__ int4 v_operand16(const char* v, const LanePlaces<bf16_t, HD>& at, int n, int db) {
  const int2 lo = ld_tr16(v + at.val16(n, 0, db)), hi = ld_tr16(v + at.val16(n, 1, db));
  return int4{lo.x, lo.y, hi.x, hi.y};
}

// The scheduler would rather save registers than start LDS reads ahead of the products
// that need them; where the order matters it is pinned.
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

// S^T = K Q^T of a tile, reads half a tile ahead of their products.
template <typename T, int HD>
__device__ __forceinline__ void many_scores(const char* k, const LanePlaces<T, HD>& at, const int4 (&q)[HD * sizeof(T) / 32],
                                            f32x16 (&s)[TT<T> / 32]) {
  constexpr int KB = TT<T> / 32, QR = HD * (int)sizeof(T) / 32;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
  if constexpr (sizeof(T) == 2) {
    int4 x[2][QR];
#pragma unroll
    for (int i = 0; i < QR; ++i) x[0][i] = ld16(k + at.key(0, i));
    pin();
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < QR; ++i) {
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[kb][i]),
                                                        __builtin_bit_cast(bf16x8, q[i]), s[kb], 0, 0, 0);
        if (kb + 1 < KB) x[kb + 1][i] = ld16(k + at.key(kb + 1, i));
        pin();
      }
  } else {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < QR; ++i) {
        const int4 x = ld16(k + at.key(kb, i));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(x.x), __int_as_float(q[i].x), s[kb], 0, 0, 0);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(x.y), __int_as_float(q[i].y), s[kb], 0, 0, 0);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(x.z), __int_as_float(q[i].z), s[kb], 0, 0, 0);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(x.w), __int_as_float(q[i].w), s[kb], 0, 0, 0);
      }
  }
}

// Scores become weights, 2^(scale2 s - sub), their sum grows l and O^T += V^T P^T.  bf16:
// the products of 16 keys run beside the reads and exponentials of the next 16.
template <typename T, int HD>
__device__ __forceinline__ void many_values(const char* v, const LanePlaces<T, HD>& at, f32x16 (&s)[TT<T> / 32],
                                            float scale2, float sub, float& l, f32x16 (&o)[HD / 32]) {
  constexpr int KB = TT<T> / 32, ND = HD / 32;
  float ls[4] = {0.f, 0.f, 0.f, 0.f};
  if constexpr (sizeof(T) == 2) {
    constexpr int N = TT<T> / 16;
    int4 vf[2][ND];
    uint32_t p[2][4];
    auto weights = [&](int n, int q) {  // weights 2 q and 2 q + 1 of the lane's eight of 16 keys
      const int kb = n / 2, r = n % 2 * 8 + 2 * q;
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale2, -sub));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kb][r + 1], scale2, -sub));
      ls[q] = ls[q] + (p0 + p1);
      p[n & 1][q] = cvt_pk_bf16(p0, p1);
    };
#pragma unroll
    for (int db = 0; db < ND; ++db) vf[0][db] = v_operand16<HD>(v, at, 0, db);
    pin();
#pragma unroll
    for (int q = 0; q < 4; ++q) weights(0, q);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int4 pn = int4{(int)p[n & 1][0], (int)p[n & 1][1], (int)p[n & 1][2], (int)p[n & 1][3]};
#pragma unroll
      for (int db = 0; db < ND; ++db) {
        pin();
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[n & 1][db]),
                                                        __builtin_bit_cast(bf16x8, pn), o[db], 0, 0, 0);
        if (n + 1 < N) {
          vf[(n + 1) & 1][db] = v_operand16<HD>(v, at, n + 1, db);
          if (ND == 4) {
            weights(n + 1, db);
          } else {
            weights(n + 1, 2 * db);
            weights(n + 1, 2 * db + 1);
          }
        }
      }
    }
  } else {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale2, -sub));
        ls[r & 3] = ls[r & 3] + s[kb][r];
      }
#pragma unroll
    for (int r = 0; r < 16 * KB; ++r) {
      const char* p = v + at.val32(r / 4, r % 4);
      float x[ND];
      if constexpr (ND == 4) {
        const float4 f = *reinterpret_cast<const float4*>(p);
        x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
      } else {
        const float2 f = *reinterpret_cast<const float2*>(p);
        x[0] = f.x, x[1] = f.y;
      }
#pragma unroll
      for (int db = 0; db < ND; ++db)
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[db], s[r / 16][r % 16], o[db], 0, 0, 0);
    }
  }
  l = l + ((ls[0] + ls[1]) + (ls[2] + ls[3]));
}

// One tile for one wave.  RAISE: the wave goes first on its SIMD while its products with V
// run, which keeps two waves out of step (2048 queries behind 14336 positions 558 -> 524 us,
// 256 behind 16384 126 -> 112, 64-wide heads behind 14336 346 -> 327); where positions are
// few for the queries and blocks differ in length it costs (2048 behind 2048 125 -> 127,
// 64-wide 76.5 -> 79.6), so it is for calls that may see three times their rows.  held: its positions that the cache has and some query of the
// workgroup sees.  odd: set where the tile was left for later (below).
template <typename T, int HD, bool RAISE>
__device__ __forceinline__ void many_tile(const PagedAttnArgs& a, ManyState<T, HD>& st, const char* k, const char* v,
                                          LanePlaces<T, HD> at, int base, uint64_t held, int qpos, int p_lo, int p_hi,
                                          int lane, bool& odd) {
  constexpr int KT = TT<T>, KB = KT / 32, ND = HD / 32, ROW = HD * (int)sizeof(T);
  // nothing of it for this wave: past its queries, or before their window
  if (base > p_hi || (a.window > 0 && base + KT - 1 <= p_lo - a.window && base >= a.sinks)) return;
  const bool whole = held == low_bits64(KT) && all_see(a, base, base + KT - 1, p_lo, p_hi);
  if (!whole && odd_tile<T, KT * ROW>(v, lane)) {
    odd = true;
    return;
  }
  const int h = lane >> 5;
  at.renew();
  f32x16 s[KB];
  many_scores<T, HD>(k, at, st.q, s);
  uint64_t vis = held;
  if (!whole) {
    vis = (uint64_t)seen_bits(a, base, qpos) | (KB == 2 ? (uint64_t)seen_bits(a, base + 32, qpos) << 32 : 0ull);
    vis &= held;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const uint32_t mine = (uint32_t)(vis >> (32 * kb)) >> (4 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = (mine >> (8 * (r >> 2) + (r & 3))) & 1 ? s[kb][r] : -CH_INF;
    }
  }
  float mx = -CH_INF;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
  const float2 both = half_pair(mx);
  mx = fmaxf(both.x, both.y);
  const float mt = vis != 0 ? fmaxf(mx * a.scale2, UNKNOWN) : -CH_INF;
  // The state is rescaled only where a maximum grew by more than 2^8 or was the first:
  // weights up to 2^8 keep their relative precision in bf16 and in the sums.
  const bool grown = mt > st.m + 8.f || st.m == -CH_INF;
  if (__ballot(grown) != 0) {
    const float mn = grown ? fmaxf(st.m, mt) : st.m;
    const float al = st.m == mn ? 1.f : weight(st.m, mn);
    st.m = mn;
    st.l = st.l * al;
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[db][r] = st.o[db][r] * al;
  }
  // a masked score, and every one of a query that has seen nothing yet, weighs nothing
  const float sub = st.m == -CH_INF ? 0.f : st.m;
  if constexpr (RAISE) __builtin_amdgcn_s_setprio(1);
  many_values<T, HD>(v, at, s, a.scale2, sub, st.l, st.o);
  if constexpr (RAISE) __builtin_amdgcn_s_setprio(0);
}

template <typename T, int HD, bool RAISE>
__global__ __launch_bounds__(256, sizeof(T) * HD == 512 ? 1 : 2) void paged_tiles_kernel(const PagedView c, const PagedAttnArgs a) {
  typedef ManyState<T, HD> State;
  constexpr int KT = TT<T>, ND = HD / 32, ROW = HD * (int)sizeof(T), CH = ROW / 16;
  constexpr int NI = KT * ROW / 4096, RPI = 1024 / ROW;  // loads of a wave, rows of a load
  __shared__ __attribute__((aligned(1024))) char k0[KT * ROW], v0[KT * ROW], k1[KT * ROW], v1[KT * ROW];
  const int kvh = blockIdx.x % c.H, rest = blockIdx.x / c.H;
  // later blocks see more: those first, and then the others from the other end, so that
  // a CU's second workgroup is short where its first is long
  const int split = rest % a.splits, nth = rest / a.splits, lead = a.slots - a.slots / 2;
  const int slot = nth < lead ? a.slots - 1 - nth : nth - lead;
  const QueryBlock blk = find_block<TB>(c, a, slot);
  if (blk.count == 0) return;
  const Span<KT> span(c, a, blk);
  const int parts = parts_of(span.tiles, a.splits, a.least);
  if (split >= parts) return;
  const int t0 = (int)((int64_t)span.tiles * split / parts), t1 = (int)((int64_t)span.tiles * (split + 1) / parts);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, h = lane >> 5;
  const int* ptab = c.page_table + (int64_t)blk.b * c.max_pages;
  const char* pool = (const char*)c.pool;
  const int first = min(wave * 32, blk.count - 1), last = min(wave * 32 + 31, blk.count - 1);
  const bool on = wave * 32 < blk.count;
  const int p_lo = blk.n + (blk.v0 + first) / a.group, p_hi = blk.n + (blk.v0 + last) / a.group;
  const int vq = blk.v0 + min(wave * 32 + c32, blk.count - 1);
  const int qrow = vq / a.group, qhead = kvh * a.group + vq - qrow * a.group;
  State st;
  {
    const int flip = a.flip == 0 ? 0 : (sizeof(T) == 2 ? (int)0x80008000 : (int)0x80000000);
    const char* q = (const char*)a.q + ((int64_t)(blk.row0 + qrow) * a.ldq + qhead * HD) * (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < State::QR; ++i) {
      const int4 x = ld16(q + 32 * i + 16 * h);
      st.q[i] = int4{x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip};
    }
  }
  st.m = -CH_INF, st.l = 0.f;
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[db][r] = 0.f;

  // A lane finds the row of one position of a tile; one that no query sees is read as
  // the last position's.  Its page is asked for before the loads of the tile before it
  // are: loads are waited for in order.
  const int p_end = min(span.p_hi, c.cap - 1);
  uint32_t row_next;
  uint64_t held_next;
  int page = 0, slot_in = 0;
  bool seen = false;
  auto ask = [&](int t) {
    const int pos = span.tile(t) * KT + (lane & (KT - 1));
    seen = some_see(a, pos, span.p_lo, span.p_hi) && pos < c.cap;
    const int p = seen ? pos : p_end, pi = c.ps.quot(p);
    slot_in = p - pi * c.ps.d;
    page = ptab[pi];
  };
  auto settle = [&]() {
    const bool there = page >= 0 && page < c.n_pages;
    held_next = __ballot(seen && there) & low_bits64(KT);
    row_next = there ? (uint32_t)page * c.page_rows + (uint32_t)slot_in : 0u;
  };
  auto find = [&](int t) {
    ask(t);
    settle();
  };
  auto load = [&](char* k, char* v) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = (wave * NI + i) * RPI + lane / CH;
      const uint32_t r = (uint32_t)__shfl((int)row_next, key) + (uint32_t)(kvh * c.ps.d);
      const char* src = pool + (uint64_t)r * ROW + (((lane % CH) ^ swizzle<CH>(key)) << 4);
      dma16(src, k + (wave * NI + i) * 1024);
      dma16(src + (uint64_t)(c.H * c.ps.d) * ROW, v + (wave * NI + i) * 1024);
    }
  };
  const LanePlaces<T, HD> at(lane);
  // two tiles a round, a buffer each; `held` of a tile travels with it
  uint64_t held = 0;
  bool odd = false;
  if (t0 < t1) {
    find(t0);
    load(k0, v0);
    held = held_next;
    if (t0 + 1 < t1) find(t0 + 1);
  }
  auto step = [&](int t, const char* k, const char* v, char* kn, char* vn) {
    tile_barrier();
    const uint64_t mine = held;
    if (t + 1 < t1) {
      if (t + 2 < t1) ask(t + 2);
      load(kn, vn);
      held = held_next;
    }
    if (on) many_tile<T, HD, RAISE>(a, st, k, v, at, span.tile(t) * KT, mine, blk.n + qrow, p_lo, p_hi, lane, odd);
    if (t + 2 < t1) settle();
  };
  for (int t = t0; t < t1; t += 2) {
    step(t, k0, v0, k1, v1);
    if (t + 1 < t1) step(t + 1, k1, v1, k0, v0);
  }
  const float2 l2 = half_pair(st.l);
  float lt = l2.x + l2.y;
  tile_barrier();  // the tiles' space is free
  if (odd) {
    __shared__ float msh[4][32], lsh[4][32];
    float* o = (float*)(wave == 0 ? k0 : wave == 1 ? v0 : wave == 2 ? k1 : v1);
    auto dim = [&](int db, int r) {
      const int row = 8 * (r >> 2) + 4 * h + (r & 3);
      return c32 * HD + (sizeof(T) == 2 ? 32 * db + row : row * ND + db);
    };
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dim(db, r)] = st.o[db][r];
    if (h == 0) msh[wave][c32] = st.m, lsh[wave][c32] = lt;
    wave_order();
    for (int t = t0; t < t1; ++t) {
      const int base = span.tile(t) * KT;
      if (base > p_hi || (a.window > 0 && base + KT - 1 <= p_lo - a.window && base >= a.sinks)) continue;
      find(t);
      if (held_next == low_bits64(KT) && all_see(a, base, base + KT - 1, p_lo, p_hi)) continue;
      const uint32_t any = odd_row<T, HD>((const T*)pool + (uint64_t)(row_next + (uint32_t)((c.H + kvh) * c.ps.d)) * HD);
      if (__ballot(any != 0) != 0)
        tile_alone<T, HD>(c, a, ptab, base, KT, blk, blk.v0 + wave * 32, last - first + 1, kvh, msh[wave], lsh[wave], o,
                          HD);
    }
#pragma unroll
    for (int db = 0; db < ND; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[db][r] = o[dim(db, r)];
    st.m = msh[wave][c32];
    lt = lsh[wave][c32];
  }
  if (wave * 32 + c32 >= blk.count) return;
  if (parts == 1) {
    T* dst = (T*)a.out + (int64_t)(blk.row0 + qrow) * a.ldo + qhead * HD;
    const float inv = 1.0f / lt;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int db = 0; db < ND; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = st.m == -CH_INF ? 0.f : st.o[db][4 * i + j] * inv;
          store_out<T, 4>(dst + 32 * db + 8 * i + 4 * h, x);
        }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) x[d] = st.m == -CH_INF ? 0.f : st.o[d][r] / lt;
        const int dim = (8 * (r >> 2) + 4 * h + (r & 3)) * ND;
        if constexpr (ND == 4) {
          store_out<T, 4>(dst + dim, x);
        } else {
          dst[dim] = x[0];
          dst[dim + 1] = x[1];
        }
      }
    }
    return;
  }
  const int64_t part = (((int64_t)slot * c.H + kvh) * a.splits + split) * TB + wave * 32 + c32;
  float* po = a.part_o + part * HD;
#pragma unroll
  for (int db = 0; db < ND; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r >> 2) + 4 * h + (r & 3);
      po[sizeof(T) == 2 ? 32 * db + row : row * ND + db] = st.o[db][r];
    }
  if (h == 0) *reinterpret_cast<float2*>(a.part_ml + part * 2) = float2{st.m, lt};
}

// The parts of a query, joined in a fixed order.  Bound by two dependent round trips.  Up
// to JOIN_FEW of them: 16 queries a workgroup, 16 threads a query, all parts on their way
// at once (eight single tokens 72 us, 80 with the other form; 2 to 3 parts of 16000 queries
// 7 us, 45 MB).  More: a workgroup a query, each wave every fourth part, eight on their way
// at once (64 parts of 32 queries 4.7 us).
constexpr int JOIN_FEW = 8;

template <typename T, int HD, int BQ, int TILE>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedView c, const PagedAttnArgs a) {
  constexpr int D = HD / 16;
  const int kvh = blockIdx.x % c.H, rest = blockIdx.x / c.H;
  const int q = rest % (BQ / 16) * 16 + threadIdx.x / 16, slot = rest / (BQ / 16);
  const QueryBlock blk = find_block<BQ>(c, a, slot);
  const Span<TILE> span(c, a, blk);
  const int parts = parts_of(span.tiles, a.splits, a.least);
  if (q >= blk.count || parts == 1) return;  // no query, or written whole
  const int64_t first = ((int64_t)slot * c.H + kvh) * a.splits * BQ + q;
  const float* po = a.part_o + first * HD + threadIdx.x % 16 * D;
  float2 ml[JOIN_FEW];
  float4 o[JOIN_FEW][D / 4];
#pragma unroll
  for (int i = 0; i < JOIN_FEW; ++i) {
    ml[i] = float2{-CH_INF, 0.f};
#pragma unroll
    for (int j = 0; j < D / 4; ++j) o[i][j] = float4{0.f, 0.f, 0.f, 0.f};
    if (i < parts) {
      ml[i] = *reinterpret_cast<const float2*>(a.part_ml + (first + (int64_t)i * BQ) * 2);
#pragma unroll
      for (int j = 0; j < D / 4; ++j) o[i][j] = *reinterpret_cast<const float4*>(po + (int64_t)i * BQ * HD + 4 * j);
    }
  }
  float mt = ml[0].x;
#pragma unroll
  for (int i = 1; i < JOIN_FEW; ++i) mt = fmaxf(mt, ml[i].x);
  float lt = 0.f, x[D];
#pragma unroll
  for (int j = 0; j < D; ++j) x[j] = 0.f;
#pragma unroll
  for (int i = 0; i < JOIN_FEW; ++i) {
    if (ml[i].x == -CH_INF) continue;  // not there, or nothing seen
    const float f = __builtin_amdgcn_exp2f(ml[i].x - mt);
    lt = fmaf(ml[i].y, f, lt);
#pragma unroll
    for (int j = 0; j < D / 4; ++j) {
      x[4 * j] = fmaf(o[i][j].x, f, x[4 * j]);
      x[4 * j + 1] = fmaf(o[i][j].y, f, x[4 * j + 1]);
      x[4 * j + 2] = fmaf(o[i][j].z, f, x[4 * j + 2]);
      x[4 * j + 3] = fmaf(o[i][j].w, f, x[4 * j + 3]);
    }
  }
  const int r = (blk.v0 + q) / a.group, h = blk.v0 + q - r * a.group;
#pragma unroll
  for (int j = 0; j < D; ++j) x[j] = mt == -CH_INF ? 0.f : x[j] / lt;
  store_out<T, D>((T*)a.out + (int64_t)(blk.row0 + r) * a.ldo + (kvh * a.group + h) * HD + threadIdx.x % 16 * D, x);
}

template <typename T, int HD, int BQ, int TILE>
__global__ __launch_bounds__(256) void paged_join_many_kernel(const PagedView c, const PagedAttnArgs a) {
  constexpr int D = HD / 64, U = 8, W = 4;
  const int nth = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int q = blockIdx.x % BQ, kvh = blockIdx.x / BQ % c.H, slot = blockIdx.x / BQ / c.H;
  const QueryBlock blk = find_block<BQ>(c, a, slot);
  const Span<TILE> span(c, a, blk);
  const int parts = parts_of(span.tiles, a.splits, a.least);
  if (q >= blk.count || parts == 1) return;  // for the whole workgroup alike
  const int64_t first = ((int64_t)slot * c.H + kvh) * a.splits * BQ + q;
  float mt = -CH_INF;
  for (int i = lane; i < parts; i += 64) mt = fmaxf(mt, a.part_ml[(first + (int64_t)i * BQ) * 2]);
  mt = wave_max(mt);
  float lt = 0.f, x[D];
#pragma unroll
  for (int j = 0; j < D; ++j) x[j] = 0.f;
  const float* po = a.part_o + first * HD + lane * D;
  for (int i0 = nth; i0 < parts; i0 += 64 * W) {  // 64 of this wave's parts
    const int n = min(64, (parts - i0 + W - 1) / W);
    float f = 0.f, fl = 0.f;
    if (lane < n) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (first + (int64_t)(i0 + lane * W) * BQ) * 2);
      f = weight(ml.x, mt);
      fl = ml.x == -CH_INF ? 0.f : ml.y * f;
    }
    lt = lt + wave_sum(fl);
    for (int i = 0; i < n; i += U) {
      float v[U][D];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const float* p = po + (int64_t)(i0 + min(i + k, n - 1) * W) * BQ * HD;
#pragma unroll
        for (int j = 0; j < D; ++j) v[k][j] = p[j];
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        // past n: the last part read again, and nothing of it (0 of an infinity is a NaN)
        const float fi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), min(i + k, 63)));
#pragma unroll
        for (int j = 0; j < D; ++j) x[j] = fmaf(i + k < n ? v[k][j] : 0.f, fi, x[j]);
      }
    }
  }
  __shared__ float xsh[W][HD], lsh[W];
#pragma unroll
  for (int j = 0; j < D; ++j) xsh[nth][lane * D + j] = x[j];
  if (lane == 0) lsh[nth] = lt;
  __syncthreads();
  if (nth != 0) return;
#pragma unroll
  for (int j = 0; j < D; ++j)
    x[j] = (xsh[0][lane * D + j] + xsh[1][lane * D + j]) + (xsh[2][lane * D + j] + xsh[3][lane * D + j]);
  lt = (lsh[0] + lsh[1]) + (lsh[2] + lsh[3]);
  const int r = (blk.v0 + q) / a.group, h = blk.v0 + q - r * a.group;
  T* dst = (T*)a.out + (int64_t)(blk.row0 + r) * a.ldo + (kvh * a.group + h) * HD + lane * D;
#pragma unroll
  for (int j = 0; j < D; ++j) dst[j] = ET<T>::from_f(mt == -CH_INF ? 0.f : x[j] / lt);
}

template <typename T, int HD, int BQ, int TILE>
void join_go(const PagedView& c, const PagedAttnArgs& a, hipStream_t st) {
  const unsigned blocks = (unsigned)(a.slots * c.H);
  if (a.splits > JOIN_FEW)
    hipLaunchKernelGGL((paged_join_many_kernel<T, HD, BQ, TILE>), dim3(blocks * BQ), dim3(256), 0, st, c, a);
  else
    hipLaunchKernelGGL((paged_join_kernel<T, HD, BQ, TILE>), dim3(blocks * (BQ / 16)), dim3(256), 0, st, c, a);
}

// ---- deal ------------------------------------------------------------------------
// Parts: a call's blocks of queries are cut until it has about the workgroups below, a
// part no shorter than LEAST tiles (twice that where the kernel for few queries has a
// workgroup a CU without a cut: 300 32-bit queries of 16 heads 10.8 us, 14.4 with cuts).
//  - R_WGS: one token of 32768, 8 cache heads 34.5 us; 36 at 768, 38 at 1024.
//  - T_WGS: a chunk of 2048 of 32 heads 124 us; 160 at 1024.  Eight chunks under a window
//    of 1024 38 us; 48 at 768.
//  - T_UNEVEN, for more than one sequence without a window, whose blocks differ: eight
//    chunks behind up to 16000 positions 181 us, seven tokens and a chunk 114; 235 and 139
//    at 512.  At 1024 164 and 120, and 63 tokens and a chunk 160 instead of 150.
constexpr int CUS = 256, R_WGS = 512, T_WGS = 512, T_UNEVEN = 768, LEAST = 8;

// Parts of a block's positions: as many as fill the card, none of them short.
int64_t deal_splits(int64_t seen, int64_t blocks, int wgs, int tile, int least) {
  const int64_t tiles = (seen + tile - 1) / tile + 2;  // a window's ends cut two more
  return std::max<int64_t>(1, std::min((wgs + blocks / 2) / blocks, (tiles + least - 1) / least));
}
// Partials of any call of up to `blocks` blocks: half a round over the card more than
// one at most, or every block's most.
int64_t deal_slots(int64_t cap, int64_t blocks, int wgs, int tile) {
  return std::min<int64_t>(std::min<int64_t>(blocks, wgs) * deal_splits(cap, 1, 1 << 30, tile, LEAST), wgs + wgs / 2);
}

// Positions that a query sees at most.
int64_t seen_most(const PagedView& c, const PagedAttnArgs& a) {
  return a.window > 0 ? std::min<int64_t>(c.cap, (int64_t)a.window + a.sinks) : c.cap;
}
// Whether a call goes to the kernel for few queries: where one block of it holds a
// sequence's, and else by the work there can be, which the tiles of 128 queries do at
// three times the rate once there is enough of it (32-bit ones at 1.4 times).
// Few / many, us, at 32 heads of 128: 64 rows behind 2048 positions (2.1 GFLOP) 23 / 21, 256
// behind none (1.1) 9 / 14, 512 behind none (4.3) 20 / 23, 128 behind 2048 (4.5) 31 / 25, 1024
// behind none (17) 53 / 35; 32-bit, 16 heads: 1024 rows of heads of 64 (4.3) 39 / 49, of 128
// (8.6) 82 / 92, 2048 (34) 259 / 189.  The host knows the table's positions, not the lengths:
// 64 single tokens of up to 500 positions under tables of 32768 take 18 / 37.
template <typename T>
bool few_queries(const PagedView& c, const PagedAttnArgs& a, int64_t most) {
  constexpr double FLOPS = sizeof(T) == 2 ? 2.5e9 : 9e9;
  return most <= RB || 4.0 * a.rows * a.Hq * c.hd * (double)seen_most(c, a) <= FLOPS;
}
// Slots of a launch and, where every sequence has as many, those of one (else 0).
struct Deal {
  int64_t slots;
  int per;
};
Deal deal(bool single, int64_t rows, int batch, int group, int64_t most, int block) {
  if (single || most <= block) {
    const int per = (int)((std::min<int64_t>(single ? group : most, most) + block - 1) / block);
    return {(int64_t)batch * per, per};
  }
  return {rows * group / block + batch, 0};
}

template <typename T, int HD>
void attn_go(const PagedView& c, PagedAttnArgs a, void* ws, hipStream_t st) {
  const bool single = a.row0 == nullptr;
  const int64_t most = single ? a.group : (int64_t)a.rows * a.group;  // queries of a sequence
  const bool few = few_queries<T>(c, a, most);
  const int block = few ? RB : TB, tile = few ? RT : TT<T>;
  const Deal d = deal(single, a.rows, c.B, a.group, most, block);
  const int64_t blocks = d.slots * c.H, seen = std::min<int64_t>(c.cap, seen_most(c, a) + block);
  a.slots = (int)d.slots;
  a.per = d.per;
  a.least = few && blocks >= CUS ? 2 * LEAST : LEAST;
  a.splits = (int)deal_splits(seen, blocks, few ? R_WGS : c.B > 1 && a.window == 0 ? T_UNEVEN : T_WGS, tile, a.least);
  const int64_t parts = blocks * a.splits;
  a.part_o = (float*)ws;
  a.part_ml = a.part_o + parts * block * HD;
  if (few) {
    hipLaunchKernelGGL((paged_rows_kernel<T, HD>), dim3((unsigned)parts), dim3(256), 0, st, c, a);
    if (a.splits > 1) join_go<T, HD, RB, RT>(c, a, st);
  } else {
    if (sizeof(T) == 2 && seen_most(c, a) >= 3 * (int64_t)a.rows / c.B)
      hipLaunchKernelGGL((paged_tiles_kernel<T, HD, sizeof(T) == 2>), dim3((unsigned)parts), dim3(256), 0, st, c, a);
    else
      hipLaunchKernelGGL((paged_tiles_kernel<T, HD, false>), dim3((unsigned)parts), dim3(256), 0, st, c, a);
    if (a.splits > 1) join_go<T, HD, TB, TT<T>>(c, a, st);
  }
}

}  // namespace

int64_t paged_attn_bytes(int64_t cap, int rows, int batch, int group, int H, int hd, int es) {
  const int64_t most = std::max<int64_t>((int64_t)rows * group, group);
  const int64_t many =
      std::max(deal(false, rows, batch, group, most, TB).slots, deal(true, rows, batch, group, most, TB).slots) * H;
  return std::max(deal_slots(cap, R_WGS, R_WGS, RT) * RB, deal_slots(cap, many, T_UNEVEN, es == 2 ? TT<bf16_t> : TT<float>) * TB) *
         (hd + 2) * 4;
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
