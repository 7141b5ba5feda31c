// Paged KV cache held in 4 bits (fp4.h): rows in, rows out, and the attention
// over it.  A row (one position's K or V of one head) is head_dim / 2 bytes of
// codes, the even dimension of a pair in the low half of its byte, and
// head_dim / 32 scale bytes; code rows lie in the order [page][K | V][head][slot],
// scale rows in the same order after all code rows.  So an element offset into
// a plain cache of that order is twice a code byte's offset and 32 times a
// scale byte's.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "fp4.h"
#include "kernels.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

// Element offset of position p of sequence b (head 0, K), -1 where the cache
// has no such slot: an unknown sequence, a position outside the table, a page
// outside the pool.
__device__ __forceinline__ int64_t kv4_slot(const Kv4View& c, int b, int p) {
  if (b < 0 || b >= c.B || p < 0 || p >= c.max_pages * c.ps) return -1;
  const int page = c.page_table[(int64_t)b * c.max_pages + p / c.ps];
  if (page < 0 || page >= c.n_pages) return -1;
  return (int64_t)page * c.page_stride + (int64_t)(p % c.ps) * c.hd;
}

// A thread's place in the rows of a call: 8 values of K or V of one row; a block
// stays within a row, so its place in the cache is found once.
struct RowPiece {
  int kv, at;  // K or V, first of the 8 values in the row
  bool on;
};
__device__ __forceinline__ RowPiece row_piece(const Kv4View& c) {
  const int width = c.H * c.hd, i = (blockIdx.x * blockDim.x + threadIdx.x) * 8;
  return {i >= width, i >= width ? i - width : i, i < 2 * width};
}
__device__ __forceinline__ int64_t piece_offset(const Kv4View& c, int64_t base, const RowPiece& p) {
  const int h = c.hd == 128 ? p.at >> 7 : p.at >> 6;
  return base + ((int64_t)p.kv * c.H + h) * c.ps * c.hd + (p.at & (c.hd - 1));
}

// Rows into the cache: grid (pieces of a row, rows), the four threads of a group
// agree on its scale.  Bound by the launch for a step's rows (64 rows of 32 heads
// of 128: 3.0 us) and by bytes for a prompt's (2044 rows: 42 MB in 12.2 us, 3.5 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4View c, const T* __restrict__ k,
                                                         const T* __restrict__ v, int64_t ld,
                                                         const int* __restrict__ seq, const int* __restrict__ pos,
                                                         const int64_t* __restrict__ off, int rows) {
  const RowPiece p = row_piece(c);
  if (!p.on) return;  // groups of four threads stay whole
  for (int row = blockIdx.y; row < rows; row += gridDim.y) {
    const int64_t base = off != nullptr ? off[row] : kv4_slot(c, seq[row], pos[row]);
    float x[8];
    load8<T>((p.kv ? v : k) + row * ld + p.at, x);
    uint32_t m = amax_bits8(x);
    m = max(m, (uint32_t)dpp_mov_i<DPP_XOR1>((int)m));
    m = max(m, (uint32_t)dpp_mov_i<DPP_XOR2>((int)m));
    const uint32_t s = fp4_scale_byte(m);
    const uint32_t w = fp4_encode8(x, s);
    if (base < 0) continue;
    const int64_t e = piece_offset(c, base, p);
    *reinterpret_cast<uint32_t*>(c.codes + e / 2) = w;
    if ((threadIdx.x & 3) == 0) c.scales[e / 32] = (uint8_t)s;
  }
}

// Rows out, as values (the same rows: 3.0 and 11.8 us).
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4View c, T* __restrict__ k, T* __restrict__ v,
                                                       int64_t ld, const int* __restrict__ seq,
                                                       const int* __restrict__ pos, int rows) {
  const RowPiece p = row_piece(c);
  if (!p.on) return;
  for (int row = blockIdx.y; row < rows; row += gridDim.y) {
    const int64_t base = kv4_slot(c, seq[row], pos[row]);
    if (base < 0) continue;
    const int64_t e = piece_offset(c, base, p);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(c.codes + e / 2);
    const float s = fp4_scale(c.scales[e / 32]);
    store8<T>((p.kv ? v : k) + row * ld + p.at, w, s);
  }
}

// A layer's rows as values, for prefill attention: grid (positions / 64, 2 H,
// segments), a thread 8 values of one of 64 positions at a time.
template <typename T>
__global__ __launch_bounds__(256) void kv4_expand_kernel(const Kv4View c, const PrefillChunk ch, T* __restrict__ pool) {
  const int seg = blockIdx.z, b = ch.seq[seg], t = blockIdx.y;
  const int end = ch.p0[seg] + ch.row0[seg + 1] - ch.row0[seg];  // positions this sequence holds
  const int per = c.hd / 8;
  for (int i = threadIdx.x; i < 64 * per; i += 256) {
    const int p = blockIdx.x * 64 + i / per;
    const int64_t base = p < end ? kv4_slot(c, b, p) : (int64_t)-1;
    if (base < 0) continue;
    const int64_t e = base + (int64_t)t * c.ps * c.hd + i % per * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(c.codes + e / 2);
    Frag32<T> f;
    f.from_fp4(w, fp4_scale(c.scales[e / 32]));
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) st16(pool + e + 4 * j, f.v[j]);
  }
}

// ---------------------------------------------------------------------------
// Attention.  Query (u, h) sits at position P = n + depth(u) and sees the
// logical keys 0 .. P, position n + e being the slot of u's depth-e ancestor.
// As in the verify pass (kernels_attn.hip) the reduction depends on P alone, so
// a query has the same bits in a tree, in a chain and by itself:
//   * positions 0 .. P - 16 are committed keys that all queries of a sequence
//     share.  An MFMA pass reduces each chunk of 64 positions by itself to
//     (m, l, O); four chunks are folded in order to a group, four groups to a
//     super, and the supers in order to the whole;
//   * the last 16 positions are reduced per query, one wave each, on top.
// Who folds does not matter, so the work is dealt by its amount.  With little of
// it a workgroup takes a group, a wave a chunk, and leaves the group's partial;
// with more it takes a super, a wave a group, and leaves a quarter of the
// partials for a quarter of the prologues (kv4_supers).
// A key that one query of the shared pass does not see and another does lies in
// the first one's window, so nothing unseen is multiplied into a result.
// ---------------------------------------------------------------------------
constexpr int CHUNK = 64, WIN = 16, FAN = 4;
constexpr int GROUP = FAN * CHUNK, SUPER = FAN * GROUP;  // positions
static_assert(WIN == KV4_MAX_DEPTH + 1, "the window holds every position of a tree");

// Depth of a lane's node.
__device__ __forceinline__ int node_depth(const Kv4Tree& t, int u) {
  uint32_t w = t.depth[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) w = u / 8 == i ? t.depth[i] : w;
  return (int)(w >> (4 * (u & 7))) & 15;
}
// u's ancestor-or-self at a lane's depth e (0 .. deep, u's own; others give 0):
// every lane holds the parent of the node of its number, the walk from u is uniform.
__device__ __forceinline__ int ancestor(const Kv4Tree& t, int u, int deep, int e, int lane) {
  uint32_t w = t.parent[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) w = lane / 4 == i ? t.parent[i] : w;
  const int parent = (int)(w >> (8 * (lane & 3))) & 63;
  int node = u, mine = 0;
  for (int d = deep; d >= 0; --d) {
    mine = e == d ? node : mine;
    node = __builtin_amdgcn_readlane(parent, node);
  }
  return mine;
}

__device__ __forceinline__ float exp2_from(float a, float b) {  // 2^(a - b), 0 from nothing
  return a == -CH_INF ? 0.f : __builtin_amdgcn_exp2f(a - b);
}
// (m, l, O) takes in (m2, l2, O2): l here, O = fma(O, x, O2 y) by the caller.  A
// side without visible keys has l == 0; a NaN is not one.
__device__ __forceinline__ bool fold(float& m, float& l, float m2, float l2, float& x, float& y) {
  if (l2 == 0.f) return false;
  const float mn = fmaxf(m, m2);
  x = exp2_from(m, mn);
  y = __builtin_amdgcn_exp2f(m2 - mn);
  l = fmaf(l, x, l2 * y);
  m = mn;
  return true;
}
__device__ __forceinline__ float fold_value(float o, float x, float o2, float y) { return fmaf(o, x, o2 * y); }
__device__ __forceinline__ f32x4 fold_value(f32x4 o, float x, f32x4 o2, float y) {
#pragma unroll
  for (int r = 0; r < 4; ++r) o[r] = fmaf(o[r], x, o2[r] * y);
  return o;
}

// Whether a sequence's shared positions 0 .. maxk are dealt in supers: where
// those alone give every CU a workgroup (32768 tokens, 8 cache heads, 256 of them:
// 15.8 us and a window of 7.3; as 1024 groups 14.2 and 18.3).  blocks: B x H x
// blocks of 16 queries.
__host__ __device__ __forceinline__ bool kv4_supers(int maxk, int blocks) {
  return (int64_t)blocks * (maxk / SUPER + 1) >= KV4_SUPER_WGS;
}

// A lane's quarter of a row: dimensions HD/4 g .. HD/4 (g + 1) - 1, eight codes
// a word, under one scale.  MFMA k-block ks takes its word ks, so the reduction
// over dimensions runs in an order of its own, the queries' too.  A row is named
// by the index of its first group of 32 values: 16 code bytes and one scale byte
// each, 32 bits for every pool that fits the card (the host checks).
template <int HD>
struct Quarter {
  uint32_t w[HD / 32];
  uint32_t s;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, uint32_t row, int g) {
    if constexpr (HD == 128) {
      const int4 v = ld16(codes + (uint64_t)(row + g) * 16);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
      s = scales[row + g];
    } else {
      const int2 v = *reinterpret_cast<const int2*>(codes + (uint64_t)(row + (g >> 1)) * 16 + 8 * (g & 1));
      w[0] = v.x, w[1] = v.y;
      s = scales[row + (g >> 1)];
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w[i] = 0;
    s = 0;
  }
};
// Queries' operand fragments in the same order of dimensions, negated for a
// negative scale: the scores' scale is then its magnitude.
template <typename T, int HD>
__device__ __forceinline__ void load_query(const T* q, int g, bool negate, Frag32<T> (&f)[HD / 32]) {
  const int flip = !negate ? 0 : (sizeof(T) == 2 ? (int)0x80008000 : (int)0x80000000);
#pragma unroll
  for (int ks = 0; ks < HD / 32; ++ks)
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) {
      const int4 v = ld16(q + (HD / 4) * g + 8 * ks + 4 * j);
      f[ks].v[j] = int4{v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip};
    }
}

// Row pitch of values staged in LDS.  16-bit V is read back transposed by
// ds_read_b64_tr_b16 (layout as in kernels_attn.hip); the pads spread the rows
// of one read over the banks.
template <typename T, int HD>
constexpr int v_pitch() { return sizeof(T) == 2 ? HD + 16 : HD + 4; }
template <typename T, int HD>
__device__ __forceinline__ void stage_quarter(const Quarter<HD>& r, T* row, int g) {
  const float sc = fp4_scale(r.s);
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    Frag32<T> f;
    f.from_fp4(r.w[i], sc);
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) st16(row + (HD / 4) * g + 8 * i + 4 * j, f.v[j]);
  }
}
__device__ __forceinline__ uint32_t cvt_pk_bf16(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}
__device__ __forceinline__ int2 ld_tr16(const void* p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
  return __builtin_bit_cast(int2, v);
}

// One chunk's scores become weights and its (m, l).  s: S^T, lane (g, c16) holding
// query c16 and keys 16 kb + 4 g + r.  vis: the chunk's keys that the query sees;
// ALL: every key, for every query of the wave (the masked path computes the same
// values then).  scale2 >= 0.  A scaled score past the float's range is an infinity:
// a chunk of nothing but negative ones (UNKNOWN, l == 1) counts for nothing next to
// any other score, a positive one makes the row NaN.
constexpr float UNKNOWN = -__FLT_MAX__;  // the maximum of scores of -inf
template <bool ALL>
__device__ __forceinline__ void chunk_weights(f32x4 (&s)[4], float scale2, uint64_t vis, int g, float& m, float& l) {
  const uint64_t mine = ALL ? 0 : vis >> (4 * g);
  float mc = -CH_INF;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) mc = fmaxf(mc, ALL || ((mine >> (16 * kb + r)) & 1) ? s[kb][r] : -CH_INF);
  mc = rows_max(mc);
  m = ALL || vis != 0 ? fmaxf(mc * scale2, UNKNOWN) : -CH_INF;
  float ls = 0.f;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float p = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale2, -m));
      if constexpr (!ALL) p = (mine >> (16 * kb + r)) & 1 ? p : 0.f;
      s[kb][r] = p;
      ls = ls + p;
    }
  l = rows_sum(ls);
  if (__ballot(fabsf(m) >= __FLT_MAX__) != 0) {
    l = m == UNKNOWN ? l + 1.f : l;
    l = m == CH_INF ? __builtin_nanf("") : l;
  }
}

// O^T += V^T P^T over the 32 keys of half kp, staged as rows v.  A weight enters
// the bf16 MFMA as three terms, hi = bf16(p), mid = bf16(p - hi) and the rest: all
// 24 bits of the float, and 4-bit values are exact, so every product is.
template <typename T, int HD>
__device__ __forceinline__ void pv_half(const f32x4 (&s)[4], int kp, const T* v, int g, int c16, f32x4 (&o)[HD / 16]) {
  constexpr int VP = v_pitch<T, HD>();
  if constexpr (sizeof(T) == 2) {
    uint32_t ph[4], pm[4], pl[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float a0 = s[2 * kp + q / 2][2 * (q % 2)], a1 = s[2 * kp + q / 2][2 * (q % 2) + 1];
      ph[q] = cvt_pk_bf16(a0, a1);
      const float r0 = a0 - __uint_as_float(ph[q] << 16), r1 = a1 - __uint_as_float(ph[q] & 0xffff0000u);
      pm[q] = cvt_pk_bf16(r0, r1);
      pl[q] = cvt_pk_bf16(r0 - __uint_as_float(pm[q] << 16), r1 - __uint_as_float(pm[q] & 0xffff0000u));
    }
    const int4 hf = int4{(int)ph[0], (int)ph[1], (int)ph[2], (int)ph[3]};
    const int4 mf = int4{(int)pm[0], (int)pm[1], (int)pm[2], (int)pm[3]};
    const int4 lf = int4{(int)pl[0], (int)pl[1], (int)pl[2], (int)pl[3]};
    const T* vrow = v + (4 * g + (c16 >> 2)) * VP + 4 * (c16 & 3);
#pragma unroll
    for (int d2 = 0; d2 < HD / 16; d2 += 2) {
      int4 vf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int2 lo = ld_tr16(vrow + 16 * (d2 + j));
        const int2 hi = ld_tr16(vrow + 16 * VP + 16 * (d2 + j));
        vf[j] = int4{lo.x, lo.y, hi.x, hi.y};
      }
      o[d2] = mfma_kb<T>(vf[0], hf, o[d2]);
      o[d2 + 1] = mfma_kb<T>(vf[1], hf, o[d2 + 1]);
      o[d2] = mfma_kb<T>(vf[0], mf, o[d2]);
      o[d2 + 1] = mfma_kb<T>(vf[1], mf, o[d2 + 1]);
      o[d2] = mfma_kb<T>(vf[0], lf, o[d2]);
      o[d2 + 1] = mfma_kb<T>(vf[1], lf, o[d2 + 1]);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 p = s[2 * kp + h];
      const int4 pf = __builtin_bit_cast(int4, p);
#pragma unroll
      for (int db = 0; db < HD / 16; ++db) {
        const T* c = v + (16 * h + 4 * g) * VP + 16 * db + c16;
        const int4 vf = int4{__float_as_int(c[0]), __float_as_int(c[VP]), __float_as_int(c[2 * VP]),
                             __float_as_int(c[3 * VP])};
        o[db] = mfma_kb<T>(vf, pf, o[db]);
      }
    }
  }
}

// x of the lanes with bit B clear and y of those with it set, each summed over
// the pair of lanes that differ in bit B.
template <int B>
__device__ __forceinline__ float pair_reduce(float x, float y, int lane) {
  if constexpr (B == 5) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else if constexpr (B == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  } else {
    const bool up = (lane >> B) & 1;
    const float keep = up ? y : x, give = up ? x : y;
    if constexpr (B == 3) return keep + dpp_mov<DPP_ROR8>(give);
    // lane ^ 4: mirrored within 8 (lane ^ 7), then within 4 (lane ^ 3)
    return keep + dpp_mov<0x1B>(dpp_mov<DPP_MIRROR8>(give));
  }
}

// The window of one query (node u, head hq of sequence b), a wave.  Lane 4 k + j
// takes quarter j of window key k, of K for the score and of V for its share of
// the output; the shares of the 16 keys are then added over the lanes, halving
// the dimensions a lane holds with each of the four steps: the lane ends with
// dimensions HD/4 j + (HD/64) rev .., rev the bits 5, 4, 3, 2 of the lane.
// request(dim) may ask for what the shared pass left, as soon as n is known;
// shared(dim, m, l, o) hands it over, for those dimensions, while the window's
// rows are in flight.
template <typename T, int HD, class Request, class Shared>
__device__ __forceinline__ void window_query(const Kv4AttnArgs& a, int b, int u, int hq, int n, int lane,
                                             Request&& request, Shared&& shared) {
  constexpr int DPL = HD / 64, DQ = HD / 4;
  const Kv4View& c = a.c;
  const int h = hq / (a.Hq / c.H);
  const int64_t row = (int64_t)b * a.N + u;
  const int kw = lane >> 2, sub = lane & 3;
  const int dim = DQ * sub + DPL * (8 * (lane >> 5) + 4 * ((lane >> 4) & 1) + 2 * ((lane >> 3) & 1) + ((lane >> 2) & 1));
  const int deep = (int)(a.tree.depth[u / 8] >> (4 * (u & 7))) & 15, P = n + deep;
  // this lane's window key
  const int p = P - WIN + 1 + kw;
  const int anc = ancestor(a.tree, u, deep, p - n, lane);
  const int at = p < n ? p : n + anc;
  const bool in = n >= 0 && p >= 0 && at < c.max_pages * c.ps;
  const int page = in ? c.page_table[(int64_t)b * c.max_pages + (unsigned)at / (unsigned)c.ps] : -1;
  request(dim);
  Frag32<T> qf[HD / 32];
  load_query<T, HD>((const T*)a.q + row * a.ldq + hq * HD, sub, a.scale < 0.f, qf);
  const bool valid = (unsigned)page < (unsigned)c.n_pages;
  const uint32_t r = valid ? (uint32_t)((int64_t)page * (c.page_stride / 32)) +
                                 (h * c.ps + (unsigned)at % (unsigned)c.ps) * (HD / 32)
                           : 0;
  Quarter<HD> k, v;
  k.load(c.codes, c.scales, r, sub);
  v.load(c.codes + (int64_t)c.H * c.ps * HD / 2, c.scales + (int64_t)c.H * c.ps * HD / 32, r, sub);
  float m = -CH_INF, l = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  shared(dim, m, l, o);
  float acc = 0.f;
  float sc = fp4_scale(k.s);
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const f32x4 x0 = fp4_to_f32x4<0>(k.w[i], sc), x1 = fp4_to_f32x4<1>(k.w[i], sc);
    const T* q = reinterpret_cast<const T*>(qf[i].v);
#pragma unroll
    for (int t = 0; t < 8; ++t) acc = fmaf(ET<T>::to_f(q[t]), t < 4 ? x0[t & 3] : x1[t & 3], acc);
  }
  acc = acc + dpp_mov<DPP_XOR1>(acc);
  acc = acc + dpp_mov<DPP_XOR2>(acc);
  const float s = valid ? acc * (fabsf(a.scale) * LOG2E) : -CH_INF;
  const float mn = fmaxf(m, wave_max(s));
  const float alpha = __ballot(valid) != 0 ? exp2_from(m, mn) : 1.f;
  const float pe = valid ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
  l = l * alpha + wave_sum(sub == 0 ? pe : 0.f);
  if (mn == UNKNOWN) l = __builtin_nanf("");  // nothing but scores of -inf
  if (!valid) v.clear();
  sc = fp4_scale(v.s);
  float w[DQ];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const f32x4 x0 = fp4_to_f32x4<0>(v.w[i], sc), x1 = fp4_to_f32x4<1>(v.w[i], sc);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      w[8 * i + t] = pe * x0[t];
      w[8 * i + 4 + t] = pe * x1[t];
    }
  }
#pragma unroll
  for (int d = 0; d < DQ / 2; ++d) w[d] = pair_reduce<5>(w[d], w[d + DQ / 2], lane);
#pragma unroll
  for (int d = 0; d < DQ / 4; ++d) w[d] = pair_reduce<4>(w[d], w[d + DQ / 4], lane);
#pragma unroll
  for (int d = 0; d < DQ / 8; ++d) w[d] = pair_reduce<3>(w[d], w[d + DQ / 8], lane);
#pragma unroll
  for (int d = 0; d < DQ / 16; ++d) w[d] = pair_reduce<2>(w[d], w[d + DQ / 16], lane);
#pragma unroll
  for (int d = 0; d < DPL; ++d) {
    const float y = l == 0.f ? 0.f : (o[d] * alpha + w[d]) / l;  // 0: no visible key
    if (a.o_mtiles > 0)
      store_tiled<T>((T*)a.out, a.o_mtiles, (int)row, hq * HD + dim + d, y);
    else
      ((T*)a.out)[row * a.ldo + hq * HD + dim + d] = ET<T>::from_f(y);
  }
}

__device__ __forceinline__ float lane_value(float v, int lane) {  // uniform
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Partials of sequence b, cache head h, unit (group or super): one a query.
__device__ __forceinline__ int64_t part_slot(const Kv4AttnArgs& a, int b, int h, int unit, int nq) {
  return (((int64_t)b * a.c.H + h) * a.units + unit) * nq;
}

// The shared pass: grid (blocks of 16 queries x H, units, B), a wave with the
// block's queries (of the N Hq / H of a cache head, node-major) as its 16 MFMA
// columns over its chunks.  K goes from memory through the conversion into the
// MFMA, V through 32 rows of wave-private LDS for its transposition: the waves
// share nothing until their partials meet.  The next chunk's K is requested when
// the scores have taken this one's, its V when this one's is used up.  Several
// query blocks of a workgroup sharing one conversion of V, with a barrier a
// chunk, were slower: 64 nodes at 512 tokens 12.8 us against 8.0.
//
// Eight single queries of 1024 to 4096 tokens, 32 heads: 28 us, 3.2 TB/s of cache.
// Its loads alone took 21 us, and without them the conversions and the softmax (some
// 520 VALU instructions a chunk) as long; over the pass the VALU is busy 31% and the
// MFMA 12% of the time: chains of three waves a SIMD, ragged lengths.  One query of
// 32768 tokens with 8 cache heads: 16 us, a wave a SIMD and its chain of four chunks.
//
// Workgroups are dealt to the eight dies round-robin, the first grid dimension
// first: heads, whose work is equal, and a head's query blocks on the die whose
// L2 has its keys (where H is a multiple of 8).  With the groups first, die i
// took group i of every head (8 ragged sequences of 1024 to 4096 tokens, single
// queries: 60 us instead of 37).
//
// ONE: a cache that holds a single group.  The workgroup goes on with its queries'
// windows, from the partials in LDS: one launch, and no partial in memory.
template <typename T, int HD, bool ONE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 3 : 2))) void kv4_shared(
    const Kv4AttnArgs a) {
  constexpr int VP = v_pitch<T, HD>(), OP = HD + 4, QP = HD + 16 / sizeof(T);  // row pitches: V, partials, queries
  union alignas(16) Stage {
    T v[32 * VP];
    float o[16 * OP];
  };
  __shared__ Stage stage_[FAN];
  __shared__ uint32_t rows_[FAN][FAN * CHUNK];
  __shared__ float ml[FAN][16][2];
  __shared__ __attribute__((aligned(16))) T qs[16 * QP];  // registers are what bounds the waves a SIMD holds
  const Kv4View& cv = a.c;
  const int h = blockIdx.x % cv.H, q0 = 16 * (blockIdx.x / cv.H), b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int n = min(a.n_b[b], cv.max_pages * cv.ps);
  const int gq = a.Hq / cv.H, nq = a.N * gq;
  const int qi = min(q0 + c16, nq - 1), u = qi / gq;
  Frag32<T> qf[HD / 32];  // one wave brings the queries
  if (wave == 0)
    load_query<T, HD>((const T*)a.q + ((int64_t)b * a.N + u) * a.ldq + (h * gq + qi % gq) * HD, g, a.scale < 0.f, qf);
  const int maxk = n < 0 ? -1 : n + a.deepest - WIN;  // last position any query treats as shared
  if (!ONE && maxk < 0) return;                       // uniform
  const bool supers = !ONE && kv4_supers(maxk, a.blocks);
  const int nu = ONE ? 1 : maxk / (supers ? SUPER : GROUP) + 1, per = supers ? FAN : 1;  // chunks a wave
  const int lim = n + node_depth(a.tree, u) - WIN;                             // this column's last shared position
  const uint8_t* vcodes = cv.codes + (int64_t)cv.H * cv.ps * HD / 2;
  const uint8_t* vscales = cv.scales + (int64_t)cv.H * cv.ps * HD / 32;
  const int* ptab = cv.page_table + (int64_t)b * cv.max_pages;
  const float scale2 = fabsf(a.scale) * LOG2E;
  T* const v = stage_[wave].v;
  uint32_t* const rows = rows_[wave];
  // page ids of a unit's keys for this wave, a lane a key: -1 past maxk
  int page[FAN];
  auto load_pages = [&](int unit) {
#pragma unroll
    for (int i = 0; i < FAN; ++i) {
      const int p = ((unit * FAN + wave) * per + i) * CHUNK + lane;
      page[i] = i < per && p <= maxk ? ptab[(unsigned)p / (unsigned)cv.ps] : -1;
    }
  };
  load_pages(blockIdx.y);
  if (wave == 0) {
#pragma unroll
    for (int ks = 0; ks < HD / 32; ++ks)
#pragma unroll
      for (int j = 0; j < (int)sizeof(T) / 2; ++j) st16(qs + c16 * QP + (HD / 4) * g + 8 * ks + 4 * j, qf[ks].v[j]);
  }
  __syncthreads();

  for (int unit = blockIdx.y; unit < nu; unit += gridDim.y) {
    const int c0 = (unit * FAN + wave) * per;
    const int nc = maxk < 0 ? 0 : min(per, maxk / CHUNK - c0 + 1);  // chunks with shared keys; may be <= 0
    float m = -CH_INF, l = 0.f;
    f32x4 o[HD / 16];
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (nc > 0) {
      // where the chunks' keys lie, a lane a key; keys past maxk and those the
      // cache does not have read group 0 and count as bad
      uint64_t bad[FAN];
#pragma unroll
      for (int i = 0; i < FAN; ++i) {
        const bool have = (unsigned)page[i] < (unsigned)cv.n_pages;
        bad[i] = __ballot(!have);
        const unsigned slot = (unsigned)((c0 + i) * CHUNK + lane) % (unsigned)cv.ps;
        if (i < per)
          rows[i * CHUNK + lane] =
              have ? (uint32_t)((int64_t)page[i] * (cv.page_stride / 32)) + (h * cv.ps + slot) * (HD / 32) : 0;
      }
      __builtin_amdgcn_wave_barrier();
      if (unit + (int)gridDim.y < nu) load_pages(unit + gridDim.y);
      Quarter<HD> k[4], vq[4];
      auto load_k = [&](int i) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) k[kb].load(cv.codes, cv.scales, rows[i * CHUNK + 16 * kb + c16], g);
      };
      auto load_v = [&](int i, int j) { vq[j].load(vcodes, vscales, rows[i * CHUNK + 16 * j + c16], g); };
      load_k(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) load_v(0, j);
      for (int i = 0; i < nc; ++i) {
        const uint64_t gone = i == 0 ? bad[0] : (i == 1 ? bad[1] : (i == 2 ? bad[2] : bad[3]));
        f32x4 s[4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < HD / 32; ++ks) {
          Frag32<T> q;
#pragma unroll
          for (int j = 0; j < (int)sizeof(T) / 2; ++j) q.v[j] = ld16(qs + c16 * QP + (HD / 4) * g + 8 * ks + 4 * j);
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) {
            Frag32<T> f;
            f.from_fp4(k[kb].w[ks], fp4_scale(k[kb].s));
            s[kb] = mfma32<T>(f, q, s[kb]);
          }
        }
        if (i + 1 < nc) load_k(i + 1);
        const int last = lim - (c0 + i) * CHUNK;  // the query's last key of the chunk
        const uint64_t vis = (last < 0 ? 0 : (last >= CHUNK - 1 ? ~0ull : (2ull << last) - 1)) & ~gone;
        float mc, lc;
        if (__ballot(vis != ~0ull) == 0)
          chunk_weights<true>(s, scale2, vis, g, mc, lc);
        else
          chunk_weights<false>(s, scale2, vis, g, mc, lc);
        f32x4 oc[HD / 16];
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) oc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kp = 0; kp < 2; ++kp) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            Quarter<HD>& r = vq[2 * kp + j];
            if ((gone >> (32 * kp + 16 * j + c16)) & 1) r.clear();  // adds exact zeros
            stage_quarter<T, HD>(r, v + (16 * j + c16) * VP, g);
          }
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
          pv_half<T, HD>(s, kp, v, g, c16, oc);
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        if (i + 1 < nc) {
#pragma unroll
          for (int j = 0; j < 4; ++j) load_v(i + 1, j);
        }
        float x = 1.f, y = 0.f;  // a query without keys here keeps what it has
        (void)fold(m, l, mc, lc, x, y);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[d] = fold_value(o[d], x, oc[d], y);
      }
    }
    // the waves' partials meet, in order
    float* po = stage_[wave].o;
    if (q0 + c16 < nq) {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4*>(po + c16 * OP + 16 * d + 4 * g) = o[d];
      if (g == 0) {
        ml[wave][c16][0] = m;
        ml[wave][c16][1] = l;
      }
    }
    __syncthreads();
    const int mine = min(nq - q0, 16);
    if constexpr (ONE) {
      constexpr int DPL = HD / 64;
      for (int q = wave; q < mine; q += FAN) {  // wave-uniform
        auto shared = [&](int dim, float& M, float& L, float (&O)[DPL]) {
#pragma unroll
          for (int w = 0; w < FAN; ++w) {
            float x, y;
            if (fold(M, L, ml[w][q][0], ml[w][q][1], x, y)) {
#pragma unroll
              for (int d = 0; d < DPL; ++d) O[d] = fold_value(O[d], x, stage_[w].o[q * OP + dim + d], y);
            }
          }
        };
        window_query<T, HD>(a, b, (q0 + q) / gq, h * gq + (q0 + q) % gq, n, lane, [](int) {}, shared);
      }
      return;
    }
    const int64_t base = part_slot(a, b, h, unit, nq) + q0;
    int first = tid;
    asm volatile("" : "+v"(first));  // what follows from it takes no registers of the chunks' loop
    for (int i = first; i < mine * (HD / 4); i += 256) {
      const int q = i / (HD / 4), d = i % (HD / 4) * 4;
      float M = -CH_INF, L = 0.f;
      f32x4 O = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < FAN; ++w) {
        const f32x4 p = *reinterpret_cast<const f32x4*>(stage_[w].o + q * OP + d);
        float x, y;
        if (fold(M, L, ml[w][q][0], ml[w][q][1], x, y)) O = fold_value(O, x, p, y);
      }
      *reinterpret_cast<f32x4*>(a.part_o + (base + q) * HD + d) = O;
      if (d == 0) *reinterpret_cast<float2*>(a.part_ml + (base + q) * 2) = float2{M, L};
    }
    __syncthreads();
  }
}

constexpr int WINDOW_BATCH = 32;  // partials of a query a wave holds at most

// 16 bytes a lane, 1 KiB a wave, from memory into LDS.
__device__ __forceinline__ void dma_1k(const float* src, float* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// grid (ceil(Hq / 4), N, B): the window after the shared pass's partials, a wave a
// query.  The partials go straight to LDS, `batch` of them a round trip.  Unrolled
// over registers, 32 of them were 27 KB of code and folds of dependent exponentials;
// now the lanes find all factors at once and a short loop multiplies and adds (one
// query of 32768 tokens, 32 partials: 12.4 -> 7.3 us).  Dependent round trips (n,
// page, rows) bound it: 64 nodes of 32 heads 5.8 us, 8192 queries 12.2 (the VALU busy
// 16% and 46% of the time).
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_window(const Kv4AttnArgs a, int batch) {
  constexpr int DPL = HD / 64, LANES = HD / 4, PER = 64 / LANES;  // lanes of a partial, partials of a load
  extern __shared__ __attribute__((aligned(16))) float parts[];   // [4][batch][HD], batch a multiple of FAN
  const Kv4View& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hq = 4 * blockIdx.x + wave, u = blockIdx.y, b = blockIdx.z;
  if (hq >= a.Hq) return;  // wave-uniform
  const int gq = a.Hq / c.H, h = hq / gq, nq = a.N * gq, qi = u * gq + hq % gq;
  const int n = min(a.n_b[b], c.max_pages * c.ps);
  const int maxk = n < 0 ? -1 : n + a.deepest - WIN;
  const bool supers = maxk >= 0 && kv4_supers(maxk, a.blocks);
  // last shared position of this query
  const int lim = n < 0 ? -1 : n + ((int)(a.tree.depth[u / 8] >> (4 * (u & 7))) & 15) - WIN;
  const int nu = lim < 0 ? 0 : lim / (supers ? SUPER : GROUP) + 1;
  const int64_t base = part_slot(a, b, h, 0, nq) + qi;
  float* const mine = parts + wave * batch * HD;
  float2 bml = float2{-CH_INF, 0.f};  // lane t: partial t of the batch
  auto load_batch = [&](int g0) {     // past the last partial: the last again
    bml = reinterpret_cast<const float2*>(a.part_ml)[base + (int64_t)min(g0 + lane, nu - 1) * nq];
    const int count = min(nu - g0, batch);
#pragma unroll 2
    for (int i = 0; i < count; i += PER)
      dma_1k(a.part_o + (base + (int64_t)min(g0 + i + lane / LANES, nu - 1) * nq) * HD + 4 * (lane % LANES),
             mine + i * HD);
  };
  auto request = [&](int) {
    if (nu > 0) load_batch(0);
  };
  auto shared = [&](int dim, float& m, float& l, float (&o)[DPL]) {
    for (int g0 = 0; g0 < nu; g0 += batch) {
      if (g0 > 0) load_batch(g0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int count = min(nu - g0, batch), step = supers ? 1 : FAN;
      // The folds' factors hang on running maxima alone: every lane finds those of
      // its partial.  top: the maximum of a partial, of a super's groups then.
      const bool have = lane < count && bml.y != 0.f;
      const uint64_t on = __ballot(have);
      float top = have ? bml.x : -CH_INF, gx = 0.f, gy = 0.f;
      if (!supers) {
        float run = fmaxf(top, __shfl_up(top, 1, FAN));
        run = fmaxf(run, __shfl_up(run, 2, FAN));
        const float before = __shfl_up(run, 1, FAN);
        gx = lane % FAN == 0 ? 0.f : exp2_from(before, run);
        gy = __builtin_amdgcn_exp2f(top - run);
        top = __shfl(run, FAN - 1, FAN);
      }
      float run = top;
      for (int s = step; s < WINDOW_BATCH; s *= 2) {
        const float v = __shfl_up(run, s);
        run = lane >= s ? fmaxf(run, v) : run;
      }
      run = fmaxf(run, m);
      const float prev = __shfl_up(run, step);
      const float x = exp2_from(lane < step ? m : prev, run), y = __builtin_amdgcn_exp2f(top - run);
      m = lane_value(run, count - 1);
      float gl = l, go[DPL];  // supers: all there is; groups: a super's, none at first
#pragma unroll
      for (int d = 0; d < DPL; ++d) go[d] = o[d];
      if (!supers) {
        gl = 0.f;
#pragma unroll
        for (int d = 0; d < DPL; ++d) go[d] = 0.f;
      }
#pragma unroll 1
      for (int t0 = 0; t0 < count; t0 += FAN) {
        float o2[FAN][DPL];
#pragma unroll
        for (int i = 0; i < FAN; ++i)
#pragma unroll
          for (int d = 0; d < DPL; ++d) o2[i][d] = mine[(t0 + i) * HD + dim + d];
        const uint32_t here = (uint32_t)(on >> t0) & ((1 << FAN) - 1);  // uniform, as all that follows
#pragma unroll
        for (int i = 0; i < FAN; ++i) {
          if (((here >> i) & 1) == 0) continue;
          const float l2 = lane_value(bml.y, t0 + i);
          const float xt = lane_value(supers ? x : gx, t0 + i), yt = lane_value(supers ? y : gy, t0 + i);
          gl = fold_value(gl, xt, l2, yt);
#pragma unroll
          for (int d = 0; d < DPL; ++d) go[d] = fold_value(go[d], xt, o2[i][d], yt);
        }
        if (supers || here == 0) continue;  // supers: gl and go are the running sums
        const float xt = lane_value(x, t0), yt = lane_value(y, t0);
        l = fold_value(l, xt, gl, yt);
        gl = 0.f;
#pragma unroll
        for (int d = 0; d < DPL; ++d) {
          o[d] = fold_value(o[d], xt, go[d], yt);
          go[d] = 0.f;
        }
      }
      if (supers) {
        l = gl;
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[d] = go[d];
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next batch comes
    }
  };
  window_query<T, HD>(a, b, u, hq, n, lane, request, shared);
}

template <typename T, int HD>
void kv4_attn_go(const Kv4AttnArgs& a, hipStream_t st) {
  const int x = a.c.H * ((a.N * (a.Hq / a.c.H) + 15) / 16);
  // A workgroup walks the units of its place.  Three a CU are resident; more only
  // cost their start, 5 to 8 ns each, where a long table holds short sequences.
  const int y = std::min(a.units, std::max(1, 2048 / (x * a.c.B)));
  if (a.one) {
    hipLaunchKernelGGL((kv4_shared<T, HD, true>), dim3(x, 1, a.c.B), dim3(256), 0, st, a);
    return;
  }
  hipLaunchKernelGGL((kv4_shared<T, HD, false>), dim3(x, y, a.c.B), dim3(256), 0, st, a);
  const dim3 grid((a.Hq + 3) / 4, a.N, a.c.B);
  const int batch = std::min(WINDOW_BATCH, (a.units + FAN - 1) / FAN * FAN);
  hipLaunchKernelGGL((kv4_window<T, HD>), grid, dim3(256), (size_t)4 * batch * HD * sizeof(float), st, a, batch);
}

}  // namespace

// Pieces of 8 values of a row's K and V in blocks of whole waves; rows past the
// grid's limit are walked.
static void row_grid(const Kv4View& c, int rows, dim3& grid, dim3& block) {
  const int pieces = c.H * c.hd / 4, threads = std::min(256, (pieces + 63) / 64 * 64);
  block = dim3(threads);
  grid = dim3((pieces + threads - 1) / threads, std::min(rows, 65535));
}

void launch_kv4_append(int dtype, const Kv4View& c, const void* k, const void* v, int64_t ld, const int* seq,
                       const int* pos, const int64_t* off, int rows, hipStream_t st) {
  dim3 grid, block;
  row_grid(c, rows, grid, block);
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(kv4_append_kernel<bf16_t>, grid, block, 0, st, c, (const bf16_t*)k, (const bf16_t*)v, ld, seq,
                       pos, off, rows);
  else
    hipLaunchKernelGGL(kv4_append_kernel<float>, grid, block, 0, st, c, (const float*)k, (const float*)v, ld, seq, pos,
                       off, rows);
}

void launch_kv4_read(int dtype, const Kv4View& c, void* k, void* v, int64_t ld, const int* seq, const int* pos,
                     int rows, hipStream_t st) {
  dim3 grid, block;
  row_grid(c, rows, grid, block);
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(kv4_read_kernel<bf16_t>, grid, block, 0, st, c, (bf16_t*)k, (bf16_t*)v, ld, seq, pos, rows);
  else
    hipLaunchKernelGGL(kv4_read_kernel<float>, grid, block, 0, st, c, (float*)k, (float*)v, ld, seq, pos, rows);
}

void launch_kv4_expand(int dtype, const Kv4View& c, const PrefillChunk& chunk, void* pool, hipStream_t st) {
  int end = 0;
  for (int k = 0; k < chunk.n_seg; ++k) end = std::max(end, chunk.p0[k] + chunk.row0[k + 1] - chunk.row0[k]);
  const dim3 grid((end + 63) / 64, 2 * c.H, chunk.n_seg);
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(kv4_expand_kernel<bf16_t>, grid, dim3(256), 0, st, c, chunk, (bf16_t*)pool);
  else
    hipLaunchKernelGGL(kv4_expand_kernel<float>, grid, dim3(256), 0, st, c, chunk, (float*)pool);
}

int kv4_attn_blocks(int B, int Hq, int H, int N) { return B * H * ((N * (Hq / H) + 15) / 16); }

int kv4_attn_units(int64_t cap, int blocks) {
  // groups are left only by sequences of fewer than KV4_SUPER_WGS / blocks supers
  const int64_t supers = (cap + SUPER - 1) / SUPER, groups = (cap + GROUP - 1) / GROUP;
  return (int)std::max(supers, std::min<int64_t>(groups, FAN * (int64_t)((KV4_SUPER_WGS + blocks - 1) / blocks)));
}

bool kv4_attn_one(int64_t cap) { return cap <= GROUP; }

int64_t kv4_attn_bytes(int B, int64_t cap, int Hq, int H, int hd, int N) {
  return (int64_t)B * kv4_attn_units(cap, kv4_attn_blocks(B, Hq, H, N)) * N * Hq * (hd + 2) * 4;
}

void launch_kv4_attn(int dtype, const Kv4AttnArgs& a, hipStream_t st) {
  if (dtype == DT_BF16 && a.c.hd == 128)
    kv4_attn_go<bf16_t, 128>(a, st);
  else if (dtype == DT_BF16)
    kv4_attn_go<bf16_t, 64>(a, st);
  else if (a.c.hd == 64)
    kv4_attn_go<float, 64>(a, st);
  else
    kv4_attn_go<float, 128>(a, st);
}
