// Verification of drafted tokens against the target's probabilities from given
// random numbers, and the next token (accept.h).
//
// p = softmax(z / T) of a row is needed at a few tokens and as running sums, in 64
// bits: a token's place in the running sum is decided by differences of 1e-6 and less
// at vocabularies of 10^5, which 32-bit sums would decide otherwise one draw in a
// thousand.
#include <algorithm>

#include "accept.h"
#include "common.h"
#include "kernels.h"

namespace {

// 2^(y / 32): y = n + f, |f| <= 1/2, 2^(n / 32) = 2^(n >> 5) times a table's
// entry, and Taylor's series of e^(f ln 2 / 32) up to the fifth power (the next is below
// 2^-48).  A weight is exp((z - m) / T) = 2^(y / 32) with y = (z - m) 32 / (T ln 2), 0 below
// 2^-1075.  Its relative error stays below 2^-48 + |y| 2^-56, of which most is the scale's,
// as if T were off by 2^-51 of itself, and a row's weights share that.  m is a row's or a
// part's largest logit: where a weight counts |y| is below 1000 then and the error below
// 2^-46.  Sums by the table of bf16 exponentials have m = 0 and |y| up to 23700, whose own
// rounding adds 2^-44 to each weight.
__device__ const double POW32[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0};
constexpr double LN2_32[5] = {0x1.62e42fefa39efp-6, 0x1.ebfbdff82c58fp-13, 0x1.c6b08d704a0c0p-20, 0x1.3b2ab6fba4e77p-27, 0x1.5d87fe78a6731p-35};  // (ln 2 / 32)^k / k!

__device__ __forceinline__ void fill_table(double* table) {  // LDS, [32]
  if (threadIdx.x < 32) table[threadIdx.x] = POW32[threadIdx.x];
}
// by: a factor within 2^750 of 1, as a table's sums are, which joins before the power of two
// can pass the range.
__device__ __forceinline__ double pow32(double y, const double* table, double by = 1.0) {
  y = fmax(y, -70400.0);
  const double n = rint(y), f = y - n;
  const int i = (int)n;
  double p = LN2_32[4];
  p = fma(p, f, LN2_32[3]);
  p = fma(p, f, LN2_32[2]);
  p = fma(p, f, LN2_32[1]);
  p = fma(p, f, LN2_32[0]);
  const double t = table[i & 31];
  return ldexp(fma(p * f, t, t) * by, i >> 5);
}
// (z - m) 32 / (T ln 2); scale: 32 / (T ln 2), at most 2^156
__device__ __forceinline__ double exponent(float z, double m, double scale) { return ((double)z - m) * scale; }

__device__ __forceinline__ double f64_of(uint32_t lo, uint32_t hi) {
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {  // 0 from lanes that are not there
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return f64_of((uint32_t)dpp_mov_i<CTRL>((int)(uint32_t)u), (uint32_t)dpp_mov_i<CTRL>((int)(uint32_t)(u >> 32)));
}
// A uniform lane's value, without a trip through LDS.
__device__ __forceinline__ double lane_f64(double v, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Over the 64 lanes, in the same order on each.
__device__ __forceinline__ double wave_sum_f64(double v) {
  v = v + dpp_f64<DPP_XOR1>(v);
  v = v + dpp_f64<DPP_XOR2>(v);
  v = v + dpp_f64<DPP_MIRROR8>(v);
  v = v + dpp_f64<DPP_MIRROR16>(v);
  uint64_t u = (uint64_t)__double_as_longlong(v);
  auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = f64_of(lo[0], hi[0]) + f64_of(lo[1], hi[1]);
  u = (uint64_t)__double_as_longlong(v);
  lo = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  hi = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return f64_of(lo[0], hi[0]) + f64_of(lo[1], hi[1]);
}
// The sum of lanes 0 .. own: within rows of 16, then the rows before.
__device__ __forceinline__ double wave_scan_f64(double v) {
  enum { SHR1 = 0x111, SHR2 = 0x112, SHR4 = 0x114, SHR8 = 0x118 };
  v = v + dpp_f64<SHR1>(v);
  v = v + dpp_f64<SHR2>(v);
  v = v + dpp_f64<SHR4>(v);
  v = v + dpp_f64<SHR8>(v);
  const double r0 = lane_f64(v, 15), r1 = r0 + lane_f64(v, 31), r2 = r1 + lane_f64(v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return v + (row == 0 ? 0.0 : row == 1 ? r0 : row == 2 ? r1 : r2);
}

template <typename T>
__device__ __forceinline__ float logit(const void* row, int64_t i) {
  return ET<T>::to_f(((const T*)row)[i]);
}
// 16 bytes at any element: rows of an odd vocabulary start at every other one (64 chains
// over 128255 bf16 tokens 71 us, 185 an entry at a time).
typedef int at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef int at4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ int4 ld16_any(const bf16_t* p) {
  const at2 x = *reinterpret_cast<const at2*>(p);
  return int4{x.x, x.y, x.z, x.w};
}
__device__ __forceinline__ int4 ld16_any(const float* p) {
  const at4 x = *reinterpret_cast<const at4*>(p);
  return int4{x.x, x.y, x.z, x.w};
}
// Sixteen of a part's entries a lane, -inf past n.  Lane l holds entries l E + 64 E i + e of
// run i, E = 16 / sizeof(T).
template <typename T>
__device__ __forceinline__ void load_part(const T* z, int n, int lane, float (&x)[16]) {
  constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 16 / E; ++i) {
    const int v = lane * E + 64 * E * i;
    if (v + E <= n) {
      const int4 w = ld16_any(z + v);
      if constexpr (sizeof(T) == 4) {
        x[4 * i] = __int_as_float(w.x), x[4 * i + 1] = __int_as_float(w.y);
        x[4 * i + 2] = __int_as_float(w.z), x[4 * i + 3] = __int_as_float(w.w);
      } else {
        const uint32_t u[4] = {(uint32_t)w.x, (uint32_t)w.y, (uint32_t)w.z, (uint32_t)w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[E * i + 2 * k] = __uint_as_float(u[k] << 16);
          x[E * i + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x[E * i + e] = v + e < n ? ET<T>::to_f(z[v + e]) : -CH_INF;
    }
  }
}

// ---- parts of rows -----------------------------------------------------------------
// Grid (rows, groups of four parts, target | draft), a wave a part.  A NaN or +inf makes a
// part's sum NaN: such a row has no distribution.  Bound by 25 instructions an entry, most
// of them in 64 bits: 704 bf16 rows of 128256 (181 MB) 80 us, VALU busy 74%; 64 32-bit rows
// of 32000 (8 MB) 5 us.  Four parts a wave: the same times.  Many bf16 rows: below.
template <typename T>
__global__ __launch_bounds__(256) void accept_parts_kernel(const AcceptArgs a) {
  __shared__ double table[32];
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int b = row / a.N, node = row - b * a.N;
  const bool of_draft = blockIdx.z != 0;
  // nothing is drawn after a node without children
  if (of_draft && !((a.inner >> node) & 1)) return;
  const int part = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* z = of_draft ? (const T*)a.draft + (int64_t)row * a.ldd : (const T*)a.logits + (int64_t)row * a.ld;
  const int root = a.tokens[(int64_t)b * a.N];
  const int v0 = part * ACCEPT_PART;
  float x[16];
  if (part < a.parts) load_part<T>(z + v0, min(ACCEPT_PART, a.V - v0), lane, x);
  fill_table(table);
  __syncthreads();
  if (root < 0 || part >= a.parts) return;  // an empty place
  bool bad = false;
  float m = -CH_INF;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    bad = bad || !(x[k] < CH_INF);
    m = fmaxf(m, x[k]);
  }
  m = wave_max(m);
  double s = 0.0;
  if (m != -CH_INF) {
#pragma unroll
    for (int k = 0; k < 16; ++k) s = s + pow32(exponent(x[k], (double)m, a.scale), table);
  }
  if (bad) s = __builtin_nan("");
  s = wave_sum_f64(s);
  if (lane == 0) {
    const int64_t at = ((int64_t)blockIdx.z * a.B * a.N + row) * a.parts + part;
    a.part_m[at] = m;
    a.part_s[at] = s;
  }
}

// The same of bf16 rows by a table: a logit has 13 bits between 2^-25 and 2^7 in magnitude,
// and exp(z / T) of all of them stays within a double's range from T = 1/4 on.  A part
// whose logits all lie there is summed with 0 for its largest; the others as above.
// A workgroup lays the table out once and its waves take part after part, the next one's
// entries on their way while one is summed.  Bound by memory and the table's reads, 8
// instructions an entry: 704 rows of 128256 (181 MB) 40 us, 4.5 TB/s.
constexpr int TABLED = 8192;
constexpr uint32_t TABLED_UP = 26 << 7;  // takes the exponents to 4 x 32 .. 4 x 32 + 31
__global__ __launch_bounds__(1024, 8) void accept_parts_tabled_kernel(const AcceptArgs a, int64_t items) {
  __shared__ double w[TABLED], table[32];
  const int lane = threadIdx.x & 63;
  fill_table(table);
  __syncthreads();
  for (int i = threadIdx.x; i < TABLED; i += 1024) {
    const uint32_t bits = (uint32_t)(i >> 12) << 15 | ((0x4000u | (i & 0xfff)) - TABLED_UP);
    w[i] = pow32(exponent(__uint_as_float(bits << 16), 0.0, a.scale), table);
  }
  __syncthreads();
  const int64_t stride = (int64_t)gridDim.x * 16;
  const int rows = a.B * a.N;
  int4 x[2];
  bool here = false;
  auto load = [&](int64_t item) {
    const int all = (int)(item / a.parts), part = (int)(item - (int64_t)all * a.parts);
    const bool of_draft = all >= rows;
    const int row = of_draft ? all - rows : all, b = row / a.N;
    const bf16_t* z = of_draft ? (const bf16_t*)a.draft + (int64_t)row * a.ldd : (const bf16_t*)a.logits + (int64_t)row * a.ld;
    here = a.tokens[(int64_t)b * a.N] >= 0 && !(of_draft && !((a.inner >> (row - b * a.N)) & 1));
    if (!here) return;
    const int n = a.V - part * ACCEPT_PART;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int v = lane * 8 + 512 * i;
      const bf16_t* p = z + part * ACCEPT_PART + v;
      if (v + 8 <= n) {
        x[i] = ld16_any(p);
      } else {
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t one = v + k < n ? (uint32_t)p[k] : 0xff80u;
          u[k / 2] = k & 1 ? u[k / 2] | one << 16 : one;
        }
        x[i] = int4{(int)u[0], (int)u[1], (int)u[2], (int)u[3]};
      }
    }
  };
  int64_t item = (int64_t)blockIdx.x * 16 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item < items) load(item);
  for (; item < items; item += stride) {
    const uint32_t u[8] = {(uint32_t)x[0].x, (uint32_t)x[0].y, (uint32_t)x[0].z, (uint32_t)x[0].w,
                           (uint32_t)x[1].x, (uint32_t)x[1].y, (uint32_t)x[1].z, (uint32_t)x[1].w};
    const bool now = here;
    if (item + stride < items) load(item + stride);
    if (!now) continue;
    uint32_t off = 0;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // a carry between the two happens only where the lower one is out of the table
      const uint32_t c = u[i] + (TABLED_UP << 16 | TABLED_UP);
      off |= c ^ 0x40004000u;
      const char* t = (const char*)w;
      s = s + *(const double*)(t + ((c << 3 & 0x7ff8u) | (c & 0x8000u)));
      s = s + *(const double*)(t + ((c >> 13 & 0x7ff8u) | (c >> 16 & 0x8000u)));
    }
    float m = 0.f;
    if (__ballot((off & 0x70007000u) != 0) != 0) {
      float y[16];
      bool bad = false;
      m = -CH_INF;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        y[k] = __uint_as_float(k & 1 ? u[k / 2] & 0xffff0000u : u[k / 2] << 16);
        bad = bad || !(y[k] < CH_INF);
        m = fmaxf(m, y[k]);
      }
      m = wave_max(m);
      s = 0.0;
      if (m != -CH_INF) {
#pragma unroll
        for (int k = 0; k < 16; ++k) s = s + pow32(exponent(y[k], (double)m, a.scale), table);
      }
      if (bad) s = __builtin_nan("");
    }
    s = wave_sum_f64(s);
    if (lane == 0) {
      a.part_m[item] = m;
      a.part_s[item] = s;
    }
  }
}

// A row's maximum and sum out of its parts, by one wave.
__device__ __forceinline__ bool distributes(const RowSum& r) {
  return r.s > 0.0 && r.s < HUGE_VAL && r.m < (double)CH_INF;
}
__device__ __forceinline__ RowSum row_sum(const AcceptArgs& a, int64_t row, const double* table) {
  const int lane = threadIdx.x & 63;
  const int64_t at = row * a.parts;
  float m = -CH_INF;
  double s = 0.0;
  for (int i = lane; i < a.parts; i += 64) {  // 64 parts at a time, a lane's own scaled to its largest
    const float pm = a.part_m[at + i];
    const double ps = a.part_s[at + i];
    const float mn = fmaxf(m, pm);
    s = m == -CH_INF ? s : s * pow32(exponent(m, (double)mn, a.scale), table);
    s = s + (pm == -CH_INF ? ps : ps * pow32(exponent(pm, (double)mn, a.scale), table));
    m = mn;
  }
  const float mt = wave_max(m);
  s = m == -CH_INF ? s : s * pow32(exponent(m, (double)mt, a.scale), table);
  return {(double)mt, wave_sum_f64(s)};
}

// ---- the walk ----------------------------------------------------------------------
// Lane u holds node u.  From the root down: a node's children are tested in the order
// of their ids; the walk goes on at the first accepted one and ends where there is
// none.  The sums of all rows with children and all nodes' probabilities come first, so
// the walk itself touches no memory but for the row of a node without children.  Bound by
// that chain: a tree of 64 nodes over 32 parts a row 4 us.
struct WalkSpace {
  double table[32];
  RowSum rows[2][64];
  Walk walk;
};
// By WAVES waves; ends with a barrier.
template <typename T, int WAVES>
__device__ void accept_walk(const AcceptArgs& a, int b, WalkSpace& sh) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = (int64_t)b * a.N;
  const bool drawn = a.draft != nullptr;
  uint32_t pw = a.tree.parent[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) pw = lane / 4 == i ? a.tree.parent[i] : pw;
  const int parent = lane == 0 ? -1 : (int)(pw >> (8 * (lane & 3))) & 255;
  const int tok = lane < a.N ? a.tokens[row0 + lane] : -1;
  const bool named = lane > 0 && lane < a.N && tok >= 0 && tok < a.V;
  double u = 0.0;
  float zp = 0.f, zq = 0.f;
  if (wave == 0 && named) {  // on their way beside the rows' sums
    u = a.u[row0 + lane];
    zp = logit<T>((const T*)a.logits + (row0 + parent) * a.ld, tok);
    if (drawn) zq = logit<T>((const T*)a.draft + (row0 + parent) * a.ldd, tok);
  }
  const bool empty = __builtin_amdgcn_readfirstlane(tok) < 0;
  fill_table(sh.table);
  __syncthreads();
  if (!empty) {
    const int n = __popcll(a.inner);
    for (int i = wave; i < (drawn ? 2 : 1) * n; i += WAVES) {
      const int z = i >= n ? 1 : 0;
      uint64_t left = a.inner;
      for (int k = i - z * n; k > 0; --k) left &= left - 1;
      const int r = __ffsll((long long)left) - 1;
      const RowSum s = row_sum(a, z * (int64_t)a.B * a.N + row0 + r, sh.table);
      if (lane == 0) sh.rows[z][r] = s;
    }
  }
  __syncthreads();
  if (wave == 0) {
    Walk w{};
    w.node = empty ? -1 : 0;
    if (!empty) {
      double p = 0.0, q = 1.0;
      if (named) {
        const RowSum rp = sh.rows[0][parent];
        p = pow32(exponent(zp, rp.m, a.scale), sh.table) / rp.s;
        if (drawn) {
          const RowSum rq = sh.rows[1][parent];
          q = pow32(exponent(zq, rq.m, a.scale), sh.table) / rq.s;
        }
      }
      w.path = 1;
      for (;;) {
        w.rejected = 0;
        w.p = (a.inner >> w.node) & 1 ? sh.rows[0][w.node] : row_sum(a, row0 + w.node, sh.table);
        w.ok = distributes(w.p);
        if (!w.ok) break;
        const uint64_t kids = __ballot(named && parent == w.node);
        if (kids == 0) break;
        if (drawn) {
          w.q = sh.rows[1][w.node];
          w.ok = distributes(w.q);
          if (!w.ok) break;
        }
        double left = 1.0;  // the mass of what is not rejected
        int next = -1;
        for (uint64_t rest = kids; rest != 0; rest &= rest - 1) {
          const int c = __builtin_amdgcn_readfirstlane(__ffsll((long long)rest) - 1);
          const double pc = lane_f64(p, c);
          if (lane_f64(u, c) * (drawn ? lane_f64(q, c) : left) < pc) {
            next = c;
            break;
          }
          w.rejected |= 1ull << c;
          left = left - pc;
          // a sibling of the same token; below other nodes it is a token like any other
          if (parent == w.node && tok == __builtin_amdgcn_readlane(tok, c)) p = 0.0;
        }
        if (next < 0) break;
        w.node = next;
        w.depth += 1;
        w.path |= 1ull << next;
      }
    }
    if (lane == 0) sh.walk = w;
  }
  __syncthreads();
}

// ---- the next token ------------------------------------------------------------------
// Weight of an entry where a walk ended: the target's probability (times the row's sum)
// where it is not a rejected token, or what the draft leaves of it.
template <typename T>
struct Weights {
  const T *z, *zq;          // zq: nullptr without a residual
  double m, mq, scale, one, one_q;
  const double* table;
  __device__ __forceinline__ double of(float x, float xq) const {
    const double p = pow32(exponent(x, m, scale), table) * one;
    return zq == nullptr ? p : fmax(p - pow32(exponent(xq, mq, scale), table) * one_q, 0.0);
  }
  __device__ __forceinline__ double operator()(int v) const {
    return of(ET<T>::to_f(z[v]), zq == nullptr ? 0.f : ET<T>::to_f(zq[v]));
  }
};

// Drawn tokens: every part of the residual, grid (groups of RESID parts, sequences), a wave
// a part, since a workgroup a sequence would leave the card idle.  Each workgroup walks by
// itself and the first of a sequence leaves the walk for the next launch.  Bound by the
// walk's chain and 64-bit instructions, 50 an entry: 8 sequences of 32000 9 us, 64 of 128256
// 22.  Whole calls with 4, 8 or 16 parts a workgroup: 19.5, 19.8 and 22.1 us for the 8
// sequences, 71, 69 and 67 for the 64; with a launch for the walks 21.3 and 70.
constexpr int RESID = 8;  // parts of a workgroup
template <typename T>
__global__ __launch_bounds__(64 * RESID) void accept_resid_kernel(const AcceptArgs a) {
  __shared__ WalkSpace sh;
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int part = blockIdx.x * RESID + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  accept_walk<T, RESID>(a, b, sh);
  const Walk w = sh.walk;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.walks[b] = w;
  if (w.node < 0 || !w.ok || w.rejected == 0) return;
  const int v0 = part * ACCEPT_PART;
  if (v0 >= a.V) return;
  const int64_t row = (int64_t)b * a.N + w.node;
  const Weights<T> f{(const T*)a.logits + row * a.ld, (const T*)a.draft + row * a.ldd, w.p.m, w.q.m, a.scale,
                     1.0 / w.p.s, 1.0 / w.q.s, sh.table};
  float x[16], xq[16];
  const int n = min(ACCEPT_PART, a.V - v0);
  load_part<T>(f.z + v0, n, lane, x);
  load_part<T>(f.zq + v0, n, lane, xq);
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = s + f.of(x[i], xq[i]);
  s = wave_sum_f64(s);
  if (lane == 0) a.resid[(int64_t)b * a.parts + part] = s;
}

// A workgroup of 1024 a sequence: the walk, its results, and the first entry whose
// running sum passes u[0] of the whole, by parts and then within one.  Bound by its chain
// of round trips and barriers: a tree of 64 nodes 10 us with its walk, 64 chains 6.5
// without.
template <typename T>
__global__ __launch_bounds__(1024) void accept_pick_kernel(const AcceptArgs a) {
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row0 = (int64_t)b * a.N;
  const int K1 = a.K + 1;
  __shared__ WalkSpace sh;
  __shared__ int gone[64], n_gone;       // rejected tokens
  __shared__ double wave_s[16], redo[64];
  __shared__ int part_sh, first_sh[16], last_sh[16];
  __shared__ double before_sh, target_sh;
  const double u0 = a.u[row0];
  if (a.draft != nullptr && a.N > 1) {
    fill_table(sh.table);
    if (tid == 0) sh.walk = a.walks[b];
    __syncthreads();
  } else {
    accept_walk<T, 16>(a, b, sh);
  }
  const Walk w = sh.walk;
  if (tid < 64) {
    const int tok = lane < a.N ? a.tokens[row0 + lane] : -1;
    const int len = w.node < 0 ? 0 : w.depth + 1;
    if (lane < a.N && w.node >= 0 && ((w.path >> lane) & 1)) {
      const int d = __popcll(w.path & ((1ull << lane) - 1));
      if (a.path != nullptr) a.path[(int64_t)b * K1 + d] = lane;
      if (d > 0) a.new_tokens[(int64_t)b * K1 + d - 1] = tok;
    }
    for (int d = lane; d < K1; d += 64) {
      if (d >= len && a.path != nullptr) a.path[(int64_t)b * K1 + d] = -1;
      if (d >= len) a.new_tokens[(int64_t)b * K1 + d] = -1;
    }
    if (lane == 0) {
      a.n_new[b] = len;
      n_gone = a.draft == nullptr ? __popcll(w.rejected) : 0;
    }
    if (a.draft == nullptr && ((w.rejected >> lane) & 1)) gone[__popcll(w.rejected & ((1ull << lane) - 1))] = tok;
  }
  __syncthreads();
  if (w.node < 0) return;
  if (!w.ok) {
    if (tid == 0) a.new_tokens[(int64_t)b * K1 + w.depth] = a.none;
    return;
  }
  const int64_t row = row0 + w.node;
  const bool resid = a.draft != nullptr && w.rejected != 0;
  Weights<T> f{(const T*)a.logits + row * a.ld, resid ? (const T*)a.draft + row * a.ldd : nullptr, w.p.m, w.q.m, a.scale,
               resid ? 1.0 / w.p.s : 1.0, resid ? 1.0 / w.q.s : 1.0, sh.table};
  int ng = n_gone;
  const int gone_l = lane < ng ? gone[lane] : -1;  // one a lane
  auto gone_of = [&](int i) { return __builtin_amdgcn_readlane(gone_l, i); };
  // Parts that hold a rejected token are summed without it, a wave each: taking it off
  // the sum would leave rounding where it was most of it.
  const int64_t parts0 = row * a.parts;
  float pm0 = -CH_INF;
  double ps0 = 0.0;
  if (wave == 0 && lane < a.parts) {  // the first parts, on their way beside this
    pm0 = a.part_m[parts0 + lane];
    ps0 = f.zq != nullptr ? a.resid[(int64_t)b * a.parts + lane] : a.part_s[parts0 + lane];
  }
  for (int i = wave - 1; i < ng; i += 15) {
    if (wave == 0) break;
    const int v0 = gone_of(i) / ACCEPT_PART * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
    constexpr int E = 16 / (int)sizeof(T);
    float x[16];
    load_part<T>(f.z + v0, n, lane, x);
    uint32_t out = 0;  // this lane's entries that are gone
    for (int j = 0; j < ng; ++j) {
      const int r = gone_of(j) - v0;
      if (r >= 0 && r < ACCEPT_PART && lane == r / E % 64) out |= 1u << (r / (64 * E) * E + r % E);
    }
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const double one = pow32(exponent(x[k], w.p.m, a.scale), sh.table);
      s = s + ((out >> k) & 1 ? 0.0 : one);
    }
    s = wave_sum_f64(s);
    if (lane == 0) redo[i] = s;
  }
  __syncthreads();
  const double redo_l = lane < ng ? redo[lane] : 0.0;
  // The part where the running sum passes, by one wave, 64 parts at a time.  Rounding
  // may leave no weight at all behind rejections (the mass that was left was its own
  // error): then the row's own probabilities decide, of which one is not 0.
  for (int attempt = 0; attempt < 2; ++attempt) {
    if (wave == 0) {
      auto part_weight = [&](int i) {
        if (i >= a.parts) return 0.0;
        const bool kept = i < 64 && attempt == 0;
        if (f.zq != nullptr) return kept ? ps0 : a.resid[(int64_t)b * a.parts + i];
        const float pm = kept ? pm0 : a.part_m[parts0 + i];
        const double ps = kept ? ps0 : a.part_s[parts0 + i];
        double of = pm == -CH_INF ? 0.0 : pow32(exponent(pm, w.p.m, a.scale), sh.table, ps);
        // a sum of 1024 that no entry has a weight behind
        of = of < 0x1p-1064 ? 0.0 : of;
        for (int j = 0; j < ng; ++j) of = gone_of(j) / ACCEPT_PART == i ? lane_f64(redo_l, j) : of;
        return of;
      };
      const double pw0 = part_weight(lane);
      double total = wave_sum_f64(pw0);
      for (int i0 = 64; i0 < a.parts; i0 += 64) total = total + wave_sum_f64(part_weight(i0 + lane));
      const double target = (u0 > 0.0 ? u0 : 0.0) * total;
      double before = 0.0, last_before = 0.0;
      int last = -1;
      for (int i0 = 0; i0 < a.parts; i0 += 64) {
        const double pw = i0 == 0 ? pw0 : part_weight(i0 + lane);
        const double upto = before + wave_scan_f64(pw);
        const uint64_t over = __ballot(pw > 0.0 && upto > target), some = __ballot(pw > 0.0);
        const int at = over != 0 ? __ffsll((long long)over) - 1 : some != 0 ? 63 - __clzll((long long)some) : -1;
        if (at >= 0) {
          last = i0 + at;
          last_before = lane_f64(upto - pw, __builtin_amdgcn_readfirstlane(at));
        }
        if (over != 0) break;
        before = lane_f64(upto, 63);
      }
      if (lane == 0) {
        part_sh = last;
        before_sh = last_before;
        target_sh = target;
      }
    }
    __syncthreads();
    if (part_sh >= 0) break;
    __syncthreads();
    ng = 0;
    f.zq = nullptr;
    f.one = 1.0;
  }
  // within the part, an entry a thread
  static_assert(ACCEPT_PART == 1024, "an entry a thread");
  const int v = part_sh * ACCEPT_PART + tid;
  bool held = v < a.V;
  for (int j = 0; j < ng; ++j) held = held && gone_of(j) != v;
  const double x = held ? f(v) : 0.0;
  const double scan = wave_scan_f64(x);
  if (lane == 63) wave_s[wave] = scan;
  __syncthreads();
  double run = before_sh;
  for (int i = 0; i < wave; ++i) run = run + wave_s[i];
  run = run + scan;
  // the first that passes; where rounding leaves none, the last with any weight
  const int wf = wave_min_i(x > 0.0 && run > target_sh ? v : 0x7fffffff), wl = -wave_min_i(x > 0.0 ? -v : 1);
  if (lane == 0) first_sh[wave] = wf, last_sh[wave] = wl;
  __syncthreads();
  if (tid == 0) {
    int first = 0x7fffffff, lastv = -1;
    for (int i = 0; i < 16; ++i) {
      first = min(first, first_sh[i]);
      lastv = max(lastv, last_sh[i]);
    }
    a.new_tokens[(int64_t)b * K1 + w.depth] = first != 0x7fffffff ? first : lastv;
  }
}

__device__ __forceinline__ uint64_t mix(uint64_t x) {  // SplitMix64
  uint64_t z = x + 0x9e3779b97f4a7c15ull;
  z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
  z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
  return z ^ (z >> 31);
}
__device__ __forceinline__ double uniform(uint64_t seed, int b, int n, int i) {
  return (double)(mix(mix(mix(mix(seed) ^ (uint64_t)b) ^ (uint64_t)n) ^ (uint64_t)i) >> 11) * 0x1p-53;
}
__global__ void accept_uniforms_kernel(const int* __restrict__ n_b, int N, unsigned long long seed, double* u) {
  const int b = blockIdx.x, i = threadIdx.x;
  if (i < N) u[(int64_t)b * N + i] = uniform(seed, b, n_b[b], i);
}
__global__ void accept_first_kernel(const PrefillEnds e, unsigned long long seed, double* u, int* tokens) {
  const int j = threadIdx.x;
  if (j >= e.n) return;
  u[j] = uniform(seed, e.seq[j], e.len[j], 64);
  tokens[j] = 0;
}

// The table costs 3 us: 6048 parts 29 us with it and 26 without, 8064 18.9 and 18.2, 10240
// 24.5 and 25.1, 12096 32 and 35, 96768 72 and 106 (whole calls).  One workgroup a CU: 79.
constexpr int64_t TABLED_PARTS = 10000;
constexpr int TABLED_WGS = 512;  // two a CU
template <typename T>
void accept_go(const AcceptArgs& a, hipStream_t st) {
  const int rows = a.B * a.N, kinds = a.draft != nullptr ? 2 : 1;
  const int64_t items = (int64_t)rows * kinds * a.parts;
  if (sizeof(T) == 2 && items >= TABLED_PARTS && a.scale <= accept_scale(0.25f))
    hipLaunchKernelGGL(accept_parts_tabled_kernel, dim3(TABLED_WGS), dim3(1024), 0, st, a, items);
  else
    hipLaunchKernelGGL((accept_parts_kernel<T>), dim3(rows, (a.parts + 3) / 4, kinds), dim3(256), 0, st, a);
  if (a.draft != nullptr && a.N > 1)
    hipLaunchKernelGGL((accept_resid_kernel<T>), dim3((a.parts + RESID - 1) / RESID, a.B), dim3(64 * RESID), 0, st, a);
  hipLaunchKernelGGL((accept_pick_kernel<T>), dim3(a.B), dim3(1024), 0, st, a);
}
int64_t up(int64_t b) { return (b + 255) / 256 * 256; }

}  // namespace

int64_t accept_bytes(int B, int N, int V, bool drawn) {
  const int64_t parts = (V + ACCEPT_PART - 1) / ACCEPT_PART, rows = (int64_t)B * N * (drawn ? 2 : 1);
  return up(rows * parts * 8) + up(rows * parts * 4) + up(drawn ? B * parts * 8 : 0) + up(drawn ? B * sizeof(Walk) : 0);
}

void accept_carve(AcceptArgs& a, void* ws) {
  a.parts = (a.V + ACCEPT_PART - 1) / ACCEPT_PART;
  const int64_t rows = (int64_t)a.B * a.N * (a.draft != nullptr ? 2 : 1);
  char* p = (char*)ws;
  a.part_s = (double*)p;
  p += up(rows * a.parts * 8);
  a.part_m = (float*)p;
  p += up(rows * a.parts * 4);
  a.resid = (double*)p;
  p += up(a.draft != nullptr ? a.B * (int64_t)a.parts * 8 : 0);
  a.walks = (Walk*)p;
}

void launch_accept(int dtype, const AcceptArgs& a, hipStream_t st) {
  if (dtype == DT_BF16)
    accept_go<bf16_t>(a, st);
  else
    accept_go<float>(a, st);
}

void launch_accept_uniforms(const int* n_b, int B, int N, unsigned long long seed, double* u, hipStream_t st) {
  hipLaunchKernelGGL(accept_uniforms_kernel, dim3(B), dim3(64), 0, st, n_b, N, seed, u);
}
void launch_accept_first(const PrefillEnds& e, unsigned long long seed, double* u, int* tokens, hipStream_t st) {
  hipLaunchKernelGGL(accept_first_kernel, dim3(1), dim3(PREFILL_SEGS), 0, st, e, seed, u, tokens);
}
