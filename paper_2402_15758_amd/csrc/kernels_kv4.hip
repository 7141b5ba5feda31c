// Paged KV cache held in 4 bits (fp4.h): rows in, rows out, and the attention
// over it.  A row (one position's K or V of one head) is head_dim / 2 bytes of
// codes, the even dimension of a pair in the low half of its byte, and
// head_dim / 32 scale bytes; code rows lie in the order [page][K | V][head][slot],
// scale rows in the same order after all code rows.  So an element offset into
// a plain cache of that order is twice a code byte's offset and 32 times a
// scale byte's.
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

// Rows into the cache: a thread takes 8 values, the four threads of a group
// agree on its scale.  Bound by bytes; a row's 8-value pieces are read whole and
// written as whole words.
template <typename T>
__global__ __launch_bounds__(256) void kv4_append_kernel(const Kv4View c, const T* __restrict__ k,
                                                         const T* __restrict__ v, int64_t ld,
                                                         const int* __restrict__ seq, const int* __restrict__ pos,
                                                         const int64_t* __restrict__ off, int64_t rows) {
  const int per = c.H * c.hd / 8;  // pieces of a row of K (or V): a multiple of 4
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / (2 * per);
  if (row >= rows) return;  // groups of four threads stay whole
  const int piece = (int)(i % (2 * per)), kv = piece / per, at = piece % per * 8;
  const int64_t base = off != nullptr ? off[row] : kv4_slot(c, seq[row], pos[row]);
  float x[8];
  load8<T>((kv ? v : k) + row * ld + at, x);
  uint32_t m = amax_bits8(x);
  m = max(m, (uint32_t)dpp_mov_i<DPP_XOR1>((int)m));
  m = max(m, (uint32_t)dpp_mov_i<DPP_XOR2>((int)m));
  const uint32_t s = fp4_scale_byte(m);
  const uint32_t w = fp4_encode8(x, s);
  if (base < 0) return;
  const int64_t e = base + ((int64_t)kv * c.H + at / c.hd) * c.ps * c.hd + at % c.hd;
  *reinterpret_cast<uint32_t*>(c.codes + e / 2) = w;
  if ((threadIdx.x & 3) == 0) c.scales[e / 32] = (uint8_t)s;
}

// Rows out, as values.
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(const Kv4View c, T* __restrict__ k, T* __restrict__ v,
                                                       int64_t ld, const int* __restrict__ seq,
                                                       const int* __restrict__ pos, int64_t rows) {
  const int per = c.H * c.hd / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / (2 * per);
  if (row >= rows) return;
  const int piece = (int)(i % (2 * per)), kv = piece / per, at = piece % per * 8;
  const int64_t base = kv4_slot(c, seq[row], pos[row]);
  if (base < 0) return;
  const int64_t e = base + ((int64_t)kv * c.H + at / c.hd) * c.ps * c.hd + at % c.hd;
  const uint32_t w = *reinterpret_cast<const uint32_t*>(c.codes + e / 2);
  const float s = fp4_scale(c.scales[e / 32]);
  const f32x4 a = fp4_to_f32x4<0>(w, s), b = fp4_to_f32x4<1>(w, s);
  T* dst = (kv ? v : k) + row * ld + at;
#pragma unroll
  for (int j = 0; j < 8; ++j) dst[j] = ET<T>::from_f(j < 4 ? a[j & 3] : b[j & 3]);
}

// ---------------------------------------------------------------------------
// Attention.  Query (u, h) sits at position P = n + depth(u) and sees the
// logical keys 0 .. P, position n + e being the slot of u's depth-e ancestor.
// As in the verify pass (kernels_attn.hip) the reduction depends on P alone, so
// a query has the same bits in a tree, in a chain and by itself:
//   * positions 0 .. P - 16 are committed keys that all queries of a sequence
//     share: an MFMA pass over chunks of 64 positions.  A run of chunks (1 below
//     position 1024, 4 from there on) is reduced by the online softmax, four
//     runs make a group, folded in run order, and a group leaves one partial
//     (m, l, O);
//   * the last 16 positions are reduced per query, one wave each, after the
//     groups' partials are folded in group order.
// A plain key is visible to every query that could see it masked in the shared
// pass, so nothing that a query does not see is multiplied into its result.
// ---------------------------------------------------------------------------
constexpr int CHUNK = 64, WIN = 16, RUNS = 4;
constexpr int NEAR_CHUNKS = 16, FAR_RUN = 4;              // runs of one chunk below NEAR_CHUNKS
constexpr int NEAR_GROUPS = NEAR_CHUNKS / RUNS;
__host__ __device__ __forceinline__ int run_chunks(int grp) { return grp < NEAR_GROUPS ? 1 : FAR_RUN; }
__host__ __device__ __forceinline__ int first_chunk(int grp) {
  return grp < NEAR_GROUPS ? grp * RUNS : NEAR_CHUNKS + (grp - NEAR_GROUPS) * RUNS * FAR_RUN;
}
__host__ __device__ __forceinline__ int groups_of(int64_t positions) {  // that cover positions 0 .. positions - 1
  const int64_t c = (positions + CHUNK - 1) / CHUNK;
  if (c <= NEAR_CHUNKS) return (int)((c + RUNS - 1) / RUNS);
  return NEAR_GROUPS + (int)((c - NEAR_CHUNKS + RUNS * FAR_RUN - 1) / (RUNS * FAR_RUN));
}
static_assert(WIN == KV4_MAX_DEPTH + 1, "the window holds every position of a tree");

__device__ __forceinline__ float exp2_from(float a, float b) {  // 2^(a - b), 0 from nothing
  return a == -CH_INF ? 0.f : __builtin_amdgcn_exp2f(a - b);
}
// (m, l) takes in (m2, l2); o = o * x + o2 * y does the rest.  A side without
// visible keys has l == 0; a NaN is not one.
__device__ __forceinline__ bool fold(float& m, float& l, float m2, float l2, float& x, float& y) {
  if (l2 == 0.f) return false;
  const float mn = fmaxf(m, m2);
  x = exp2_from(m, mn);
  y = __builtin_amdgcn_exp2f(m2 - mn);
  l = l * x + l2 * y;
  m = mn;
  return true;
}

// A lane's quarter of a row: dimensions HD/4 g .. HD/4 (g + 1) - 1, eight codes
// a word, under one scale.  MFMA k-block ks takes its word ks, so the reduction
// over dimensions runs in an order of its own, the queries' too.
template <int HD>
struct Quarter {
  uint32_t w[HD / 32];
  uint32_t s;
  __device__ __forceinline__ void load(const Kv4View& c, int64_t e, int g) {  // e: the row's element offset
    const uint8_t* p = c.codes + e / 2 + g * (HD / 8);
    if constexpr (HD == 128) {
      const int4 v = ld16(p);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      const int2 v = *reinterpret_cast<const int2*>(p);
      w[0] = v.x, w[1] = v.y;
    }
    s = c.scales[e / 32 + g * (HD / 4) / 32];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) w[i] = 0;
    s = 0;
  }
};
// Queries' operand fragments in the same order of dimensions.
template <typename T, int HD>
__device__ __forceinline__ void load_query(const T* q, int g, Frag32<T> (&f)[HD / 32]) {
#pragma unroll
  for (int ks = 0; ks < HD / 32; ++ks)
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) f[ks].v[j] = ld16(q + (HD / 4) * g + 8 * ks + 4 * j);
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

// One chunk's scores become weights.  s: S^T, lane (g, c16) holding query c16 and
// keys 16 kb + 4 g + r.  vis: the chunk's keys that the query sees.  Updates
// (m, l) and returns the factor for O; all: every key is visible to every
// query of the wave (the masked path computes the same values then).
__device__ __forceinline__ float chunk_weights(f32x4 (&s)[4], float scale2, bool all, uint64_t vis, int g, float& m,
                                               float& l) {
  float mc = -CH_INF;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v = s[kb][r] * scale2;
      if (!all && !((vis >> (16 * kb + 4 * g + r)) & 1)) v = -CH_INF;
      s[kb][r] = v;
      mc = fmaxf(mc, v);
    }
  mc = rows_max(mc);
  const float mn = fmaxf(m, mc);
  const float alpha = vis != 0 || all ? exp2_from(m, mn) : 1.f;
  float ls = 0.f;
#pragma unroll
  for (int kb = 0; kb < 4; ++kb)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float p = __builtin_amdgcn_exp2f(s[kb][r] - mn);
      if (!all && !((vis >> (16 * kb + 4 * g + r)) & 1)) p = 0.f;
      s[kb][r] = p;
      ls = ls + p;
    }
  ls = rows_sum(ls);
  l = l * alpha + ls;
  m = mn;
  return alpha;
}

// O^T += V^T P^T over the 32 keys of half kp, staged as rows v.  A weight enters
// the bf16 MFMA as two terms, hi = bf16(p) and bf16(p - hi): 16 bits of it, a
// rounding of 2^-17, next to the 2^-9 of a bf16 output; 4-bit values are exact.
template <typename T, int HD>
__device__ __forceinline__ void pv_half(const f32x4 (&s)[4], int kp, const T* v, int g, int c16, f32x4 (&o)[HD / 16]) {
  constexpr int VP = v_pitch<T, HD>();
  if constexpr (sizeof(T) == 2) {
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float a0 = s[2 * kp + q / 2][2 * (q % 2)], a1 = s[2 * kp + q / 2][2 * (q % 2) + 1];
      ph[q] = cvt_pk_bf16(a0, a1);
      pl[q] = cvt_pk_bf16(a0 - __uint_as_float(ph[q] << 16), a1 - __uint_as_float(ph[q] & 0xffff0000u));
    }
    const int4 hf = int4{(int)ph[0], (int)ph[1], (int)ph[2], (int)ph[3]};
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

// What both shapes of the shared pass need of a workgroup: sequence b, cache
// head h, group grp.
struct SharedPart {
  int n, grp, c_begin, c_end;  // chunks of the group with visible keys
  int maxk;                    // last position any query treats as shared
};
__device__ __forceinline__ bool shared_part(const Kv4AttnArgs& a, int b, SharedPart& p) {
  p.grp = blockIdx.x;
  p.n = min(a.n_b[b], a.c.max_pages * a.c.ps);
  p.maxk = p.n < 0 ? -1 : p.n + a.deepest - WIN;
  p.c_begin = first_chunk(p.grp);
  p.c_end = min(p.c_begin + RUNS * run_chunks(p.grp) - 1, p.maxk < 0 ? -1 : p.maxk / CHUNK);
  return p.c_begin <= p.c_end;
}
// The query of lane column c16: index qi of the sequence's N Hq / H queries of a
// cache head, node-major.
template <typename T, int HD>
__device__ __forceinline__ int query_of(const Kv4AttnArgs& a, int b, int h, int qi, int n, int g,
                                        Frag32<T> (&qf)[HD / 32]) {
  const int gq = a.Hq / a.c.H, u = qi / gq;
  load_query<T, HD>((const T*)a.q + ((int64_t)b * a.N + u) * a.ldq + (h * gq + qi % gq) * HD, g, qf);
  return n + a.tree.depth[u] - WIN;  // its last shared position
}
// Keys of chunk c that a query with last shared position lim sees.
__device__ __forceinline__ uint64_t visible(int c, int lim, uint64_t bad) {
  const int k = lim - c * CHUNK;  // last visible key of the chunk
  const uint64_t in = k < 0 ? 0 : (k >= CHUNK - 1 ? ~0ull : (2ull << k) - 1);
  return in & ~bad;
}
__device__ __forceinline__ int64_t part_slot(const Kv4AttnArgs& a, int b, int h, int grp, int nq) {
  return (((int64_t)b * a.c.H + h) * a.groups + grp) * nq;
}

// Up to 16 queries a cache head (single tokens, short chains, few grouped
// heads): grid (groups, H, B), a wave takes a run of the group's chunks with
// all queries as its 16 MFMA columns.  Waves share nothing until their runs are
// done: K goes from memory through the conversion into the MFMA, V through 32
// rows of wave-private LDS for its transposition; K of the next chunk is
// requested as soon as the scores have taken this chunk's, V likewise.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_shared_few(const Kv4AttnArgs a) {
  constexpr int VP = v_pitch<T, HD>();
  __shared__ __attribute__((aligned(16))) T vs[RUNS][32 * VP];
  __shared__ int64_t slots[RUNS][CHUNK];
  __shared__ float ml[RUNS][16][2];
  static_assert(sizeof(T) * 32 * VP >= 16 * HD * 4, "a run's partial fits its staging rows");
  const Kv4View& cv = a.c;
  const int h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  SharedPart sp;
  if (!shared_part(a, b, sp)) return;  // uniform
  const int nq = a.N * (a.Hq / cv.H);
  Frag32<T> qf[HD / 32];
  const int lim = query_of<T, HD>(a, b, h, min(c16, nq - 1), sp.n, g, qf);
  const int rc = run_chunks(sp.grp), c0 = sp.c_begin + wave * rc, c1 = min(c0 + rc - 1, sp.c_end);
  const float scale2 = a.scale * LOG2E;
  float m = -CH_INF, l = 0.f;
  f32x4 o[HD / 16];
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  T* v = vs[wave];
  int64_t* sl = slots[wave];
  const int64_t head = (int64_t)h * cv.ps * HD, vofs = (int64_t)cv.H * cv.ps * HD;
  if (c0 <= c1) {  // wave-uniform
    // lane i works out key i's slot; rows past the last shared position and
    // those the cache does not have read slot 0 of page 0 and count as bad
    auto slot = [&](int c) {
      const int p = c * CHUNK + lane;
      return p <= sp.maxk ? kv4_slot(cv, b, p) : (int64_t)-1;
    };
    uint64_t bad = 0, bad_next = 0;
    auto put = [&](int64_t e) {
      sl[lane] = (e < 0 ? 0 : e) + head;
      __builtin_amdgcn_wave_barrier();
    };
    Quarter<HD> k[4], vq[4];
    int64_t e = slot(c0);
    bad = __ballot(e < 0);
    put(e);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int64_t r = sl[16 * kb + c16];
      k[kb].load(cv, r, g);
      vq[kb].load(cv, r + vofs, g);
    }
    for (int c = c0; c <= c1; ++c) {
      int64_t en = c < c1 ? slot(c + 1) : (int64_t)-1;
      f32x4 s[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const float sc = fp4_scale(k[kb].s);
        s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < HD / 32; ++ks) {
          Frag32<T> f;
          f.from_fp4(k[kb].w[ks], sc);
          s[kb] = mfma32<T>(f, qf[ks], s[kb]);
        }
      }
      if (c < c1) {
        bad_next = __ballot(en < 0);
        put(en);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) k[kb].load(cv, sl[16 * kb + c16], g);
      }
      const uint64_t vis = visible(c, lim, bad);
      const bool all = __ballot(vis != ~0ull) == 0;
      const float alpha = chunk_weights(s, scale2, all, vis, g, m, l);
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d] = o[d] * alpha;
#pragma unroll
      for (int kp = 0; kp < 2; ++kp) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          Quarter<HD>& r = vq[2 * kp + j];
          if (bad != 0 && ((bad >> (32 * kp + 16 * j + c16)) & 1)) r.clear();  // adds exact zeros
          stage_quarter<T, HD>(r, v + (16 * j + c16) * VP, g);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        pv_half<T, HD>(s, kp, v, g, c16, o);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
      if (c < c1) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) vq[kb].load(cv, sl[16 * kb + c16] + vofs, g);
      }
      bad = bad_next;
    }
  }
  // the runs meet in LDS, in run order
  float* po = reinterpret_cast<float*>(v);
  if (c16 < nq) {
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4*>(po + c16 * HD + 16 * d + 4 * g) = o[d];
    if (g == 0) {
      ml[wave][c16][0] = m;
      ml[wave][c16][1] = l;
    }
  }
  __syncthreads();
  const int64_t base = part_slot(a, b, h, sp.grp, nq);
  for (int i = tid; i < nq * HD; i += 256) {
    const int q = i / HD;
    float M = -CH_INF, L = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < RUNS; ++w) {
      float x, y;
      if (fold(M, L, ml[w][q][0], ml[w][q][1], x, y)) O = O * x + reinterpret_cast<const float*>(vs[w])[i] * y;
    }
    a.part_o[base * HD + i] = O;
    if (i % HD == 0) {
      a.part_ml[(base + q) * 2] = M;
      a.part_ml[(base + q) * 2 + 1] = L;
    }
  }
}

// More queries: grid (groups, H x blocks of 64 queries, B).  The workgroup
// converts each chunk once into LDS, the waves own 16 queries each and walk the
// chunks, folding a run at its end.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_shared_many(const Kv4AttnArgs a) {
  constexpr int VP = v_pitch<T, HD>(), KP = HD + 16 / sizeof(T);
  __shared__ __attribute__((aligned(16))) T ks_[CHUNK * KP];
  __shared__ __attribute__((aligned(16))) T vs[CHUNK * VP];
  const Kv4View& cv = a.c;
  const int h = blockIdx.y % cv.H, qb = blockIdx.y / cv.H, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  SharedPart sp;
  if (!shared_part(a, b, sp)) return;
  const int nq = a.N * (a.Hq / cv.H), qi = 64 * qb + 16 * wave + c16;
  const bool wave_on = 64 * qb + 16 * wave < nq;  // wave-uniform
  Frag32<T> qf[HD / 32];
  const int lim = query_of<T, HD>(a, b, h, min(qi, nq - 1), sp.n, g, qf);
  const int rc = run_chunks(sp.grp);
  const float scale2 = a.scale * LOG2E;
  float m = -CH_INF, l = 0.f, fm = -CH_INF, fl = 0.f;
  f32x4 o[HD / 16], fo[HD / 16];
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) o[d] = fo[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t head = (int64_t)h * cv.ps * HD, vofs = (int64_t)cv.H * cv.ps * HD;
  // thread (key, quarter) brings that quarter of K's and V's row
  const int key = tid >> 2, quarter = tid & 3;
  auto slot = [&](int c) {
    const int p = c * CHUNK + key;
    return p <= sp.maxk ? kv4_slot(cv, b, p) : (int64_t)-1;
  };
  __shared__ uint32_t bad_bits[2][4];  // of the chunk in LDS: 16 keys a wave
  Quarter<HD> k, v;
  int64_t e = slot(sp.c_begin);
  k.load(cv, (e < 0 ? 0 : e) + head, quarter);
  v.load(cv, (e < 0 ? 0 : e) + head + vofs, quarter);
  for (int c = sp.c_begin; c <= sp.c_end; ++c) {
    const int64_t en = c < sp.c_end ? slot(c + 1) : (int64_t)-1;
    const uint64_t wb = __ballot(e < 0);
    if (c > sp.c_begin) __syncthreads();  // the last chunk's readers are done
    if (e < 0) v.clear();
    stage_quarter<T, HD>(k, ks_ + key * KP, quarter);
    stage_quarter<T, HD>(v, vs + key * VP, quarter);
    if (lane == 0) {
      uint32_t x = 0;  // one bit a key: its four threads agree
#pragma unroll
      for (int i = 0; i < 16; ++i) x |= (uint32_t)((wb >> (4 * i)) & 1) << i;
      bad_bits[c & 1][wave] = x;
    }
    __syncthreads();
    if (c < sp.c_end) {
      k.load(cv, (en < 0 ? 0 : en) + head, quarter);
      v.load(cv, (en < 0 ? 0 : en) + head + vofs, quarter);
    }
    e = en;
    if (!wave_on) continue;
    const uint32_t* bb = bad_bits[c & 1];
    const uint64_t bad = (uint64_t)(bb[0] | bb[1] << 16) | (uint64_t)(bb[2] | bb[3] << 16) << 32;
    f32x4 s[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < HD / 32; ++t) {
        Frag32<T> f;
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j)
          f.v[j] = ld16(ks_ + (16 * kb + c16) * KP + (HD / 4) * g + 8 * t + 4 * j);
        s[kb] = mfma32<T>(f, qf[t], s[kb]);
      }
    }
    const uint64_t vis = visible(c, lim, bad);
    const bool all = __ballot(vis != ~0ull) == 0;
    const float alpha = chunk_weights(s, scale2, all, vis, g, m, l);
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[d] = o[d] * alpha;
#pragma unroll
    for (int kp = 0; kp < 2; ++kp) pv_half<T, HD>(s, kp, vs + 32 * kp * VP, g, c16, o);
    if (c == sp.c_end || (c + 1 - sp.c_begin) % rc == 0) {  // a run ends
      float x, y;
      if (fold(fm, fl, m, l, x, y)) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) fo[d] = fo[d] * x + o[d] * y;
      }
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
      m = -CH_INF;
      l = 0.f;
    }
  }
  if (qi >= nq) return;
  const int64_t at = part_slot(a, b, h, sp.grp, nq) + qi;
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4*>(a.part_o + at * HD + 16 * d + 4 * g) = fo[d];
  if (g == 0) {
    a.part_ml[at * 2] = fm;
    a.part_ml[at * 2 + 1] = fl;
  }
}

// The window: grid (ceil(Hq / 4), N, B), a wave per query.  Lane 4 k + j scores
// quarter j of window key k; for the output each lane reads its own dimensions
// of every row.  The groups' partials are folded while the rows are in flight.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_window(const Kv4AttnArgs a) {
  constexpr int DPL = HD / 64, BATCH = 8;
  const Kv4View& c = a.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hq = 4 * blockIdx.x + wave, u = blockIdx.y, b = blockIdx.z;
  if (hq >= a.Hq) return;  // wave-uniform
  const int gq = a.Hq / c.H, h = hq / gq, nq = a.N * gq, qi = u * gq + hq % gq;
  const int64_t row = (int64_t)b * a.N + u;
  const int kw = lane >> 2, sub = lane & 3;
  const int n = min(a.n_b[b], c.max_pages * c.ps);
  Frag32<T> qf[HD / 32];
  load_query<T, HD>((const T*)a.q + row * a.ldq + hq * HD, sub, qf);
  const int P = n + a.tree.depth[u];
  const int lim = P - WIN;
  const int ngrp = n < 0 || lim < 0 ? 0 : groups_of((int64_t)lim + 1);
  const int64_t base = part_slot(a, b, h, 0, nq) + qi;
  float bm[BATCH], bl[BATCH], bo[BATCH][DPL];
  auto load_batch = [&](int g0) {
#pragma unroll
    for (int t = 0; t < BATCH; ++t) {
      const int64_t at = base + (int64_t)min(g0 + t, ngrp - 1) * nq;
      bm[t] = a.part_ml[at * 2];
      bl[t] = a.part_ml[at * 2 + 1];
#pragma unroll
      for (int d = 0; d < DPL; ++d) bo[t][d] = a.part_o[at * HD + DPL * lane + d];
    }
  };
  if (ngrp > 0) load_batch(0);
  // this lane's window key
  const int p = P - WIN + 1 + kw;
  const int at = p < n ? p : n + a.tree.path[u][min(max(p - n, 0), KV4_MAX_DEPTH)];
  int64_t e = n >= 0 && p >= 0 ? kv4_slot(c, b, at) : (int64_t)-1;
  const bool valid = e >= 0;
  e = (valid ? e : 0) + (int64_t)h * c.ps * HD;
  const uint64_t ok = __ballot(valid);
  Quarter<HD> k;
  k.load(c, e, sub);
  uint32_t vc[WIN], vsc[WIN];
  const int64_t vofs = (int64_t)c.H * c.ps * HD + DPL * lane;
#pragma unroll
  for (int i = 0; i < WIN; ++i) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)e, 4 * i);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(e >> 32), 4 * i);
    const int64_t ve = (int64_t)((uint64_t)hi << 32 | lo) + vofs;
    vc[i] = c.codes[ve / 2];
    vsc[i] = c.scales[ve / 32];
  }
  float m = -CH_INF, l = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  for (int g0 = 0; g0 < ngrp; g0 += BATCH) {
    if (g0 > 0) load_batch(g0);
#pragma unroll
    for (int t = 0; t < BATCH; ++t) {
      float x, y;
      if (g0 + t < ngrp && fold(m, l, bm[t], bl[t], x, y)) {
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[d] = o[d] * x + bo[t][d] * y;
      }
    }
  }
  float acc = 0.f;
  const float sc = fp4_scale(k.s);
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const f32x4 x0 = fp4_to_f32x4<0>(k.w[i], sc), x1 = fp4_to_f32x4<1>(k.w[i], sc);
    const T* q = reinterpret_cast<const T*>(qf[i].v);
#pragma unroll
    for (int t = 0; t < 8; ++t) acc = fmaf(ET<T>::to_f(q[t]), t < 4 ? x0[t & 3] : x1[t & 3], acc);
  }
  acc = acc + dpp_mov<DPP_XOR1>(acc);
  acc = acc + dpp_mov<DPP_XOR2>(acc);
  const float s = valid ? acc * (a.scale * LOG2E) : -CH_INF;
  const float mn = fmaxf(m, wave_max(s));
  const float alpha = ok != 0 ? exp2_from(m, mn) : 1.f;
  const float pe = valid ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
  l = l * alpha + wave_sum(sub == 0 ? pe : 0.f);
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = o[d] * alpha;
#pragma unroll
  for (int i = 0; i < WIN; ++i) {
    if (!((ok >> (4 * i)) & 1)) continue;  // wave-uniform
    const float pk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(pe), 4 * i));
    const uint32_t w = DPL == 1 ? vc[i] >> (4 * (lane & 1)) : vc[i];
    const f32x4 x = fp4_to_f32x4<0>(w, fp4_scale(vsc[i]));
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] = fmaf(pk, x[d], o[d]);
  }
#pragma unroll
  for (int d = 0; d < DPL; ++d) {
    const float r = l == 0.f ? 0.f : o[d] / l;  // no visible key
    if (a.o_mtiles > 0)
      store_tiled<T>((T*)a.out, a.o_mtiles, (int)row, hq * HD + DPL * lane + d, r);
    else
      ((T*)a.out)[row * a.ldo + hq * HD + DPL * lane + d] = ET<T>::from_f(r);
  }
}

template <typename T, int HD>
void kv4_attn_go(const Kv4AttnArgs& a, hipStream_t st) {
  const int nq = a.N * (a.Hq / a.c.H);
  if (nq <= 16)
    hipLaunchKernelGGL((kv4_shared_few<T, HD>), dim3(a.groups, a.c.H, a.c.B), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((kv4_shared_many<T, HD>), dim3(a.groups, a.c.H * ((nq + 63) / 64), a.c.B), dim3(256), 0, st, a);
  hipLaunchKernelGGL((kv4_window<T, HD>), dim3((a.Hq + 3) / 4, a.N, a.c.B), dim3(256), 0, st, a);
}

}  // namespace

void launch_kv4_append(int dtype, const Kv4View& c, const void* k, const void* v, int64_t ld, const int* seq,
                       const int* pos, const int64_t* off, int64_t rows, hipStream_t st) {
  const dim3 grid((unsigned)((rows * (c.H * c.hd / 4) + 255) / 256));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(kv4_append_kernel<bf16_t>, grid, dim3(256), 0, st, c, (const bf16_t*)k, (const bf16_t*)v, ld,
                       seq, pos, off, rows);
  else
    hipLaunchKernelGGL(kv4_append_kernel<float>, grid, dim3(256), 0, st, c, (const float*)k, (const float*)v, ld, seq,
                       pos, off, rows);
}

void launch_kv4_read(int dtype, const Kv4View& c, void* k, void* v, int64_t ld, const int* seq, const int* pos,
                     int64_t rows, hipStream_t st) {
  const dim3 grid((unsigned)((rows * (c.H * c.hd / 4) + 255) / 256));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(kv4_read_kernel<bf16_t>, grid, dim3(256), 0, st, c, (bf16_t*)k, (bf16_t*)v, ld, seq, pos, rows);
  else
    hipLaunchKernelGGL(kv4_read_kernel<float>, grid, dim3(256), 0, st, c, (float*)k, (float*)v, ld, seq, pos, rows);
}

int kv4_attn_groups(int64_t cap) { return groups_of(cap); }

int64_t kv4_attn_bytes(int B, int64_t cap, int Hq, int hd, int N) {
  return (int64_t)B * groups_of(cap) * N * Hq * (hd + 2) * 4;
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
