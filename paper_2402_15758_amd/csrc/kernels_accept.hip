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

// 2^(y / 32) for y <= 0: y = n + f, |f| <= 1/2, 2^(n / 32) = 2^(n >> 5) times a table's
// entry, and Taylor's series of e^(f ln 2 / 32) up to the fifth power (the next is below
// 2^-48).  A weight is exp((z - m) / T) = 2^(y / 32) with y = (z - m) 32 / (T ln 2): the
// sum of a row's errors stays below 2^-47 of its weights.  0 from 2^-1100 on.
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
__device__ __forceinline__ double pow32(double y, const double* table) {
  y = fmax(y, -35200.0);
  const double n = rint(y), f = y - n;
  const int i = (int)n;
  double p = LN2_32[4];
  p = fma(p, f, LN2_32[3]);
  p = fma(p, f, LN2_32[2]);
  p = fma(p, f, LN2_32[1]);
  p = fma(p, f, LN2_32[0]);
  const double t = table[i & 31];
  return ldexp(fma(p * f, t, t), i >> 5);
}
// (z - m) 32 / (T ln 2); scale: 32 / (T ln 2), at most 2^156
__device__ __forceinline__ double exponent(float z, double m, double scale) { return ((double)z - m) * scale; }

__device__ __forceinline__ double shfl_f64(double v, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return __longlong_as_double((long long)((uint64_t)(uint32_t)__shfl((int)(uint32_t)u, lane) |
                                          ((uint64_t)(uint32_t)__shfl((int)(uint32_t)(u >> 32), lane) << 32)));
}
// Over the 64 lanes, in the same order on each.
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = v + shfl_f64(v, (threadIdx.x & 63) ^ d);
  return v;
}
// The sum of lanes 0 .. own.
__device__ __forceinline__ double wave_scan_f64(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double w = shfl_f64(v, max(lane - d, 0));
    v = lane >= d ? v + w : v;
  }
  return v;
}

template <typename T>
__device__ __forceinline__ float logit(const void* row, int64_t i) {
  return ET<T>::to_f(((const T*)row)[i]);
}
// Sixteen of a part's entries a lane, -inf past n; VEC: 16 bytes at once.  Lane l holds
// entries l * E + 64 E i + e of run i, E = 16 / sizeof(T) (1 without VEC).
template <typename T, bool VEC>
__device__ __forceinline__ void load_part(const T* z, int n, int lane, float (&x)[16]) {
  constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
#pragma unroll
  for (int i = 0; i < 16 / E; ++i) {
    const int v = lane * E + 64 * E * i;
    if (VEC && v + E <= n) {
      const int4 w = ld16(z + v);
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
// Grid (rows, groups of four parts, target | draft), a wave a part.  A NaN or +inf makes
// the part's sum NaN: such a row has no distribution.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void accept_parts_kernel(const AcceptArgs a) {
  __shared__ double table[32];
  fill_table(table);
  const int row = blockIdx.x, lane = threadIdx.x & 63;
  const int part = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool of_draft = blockIdx.z != 0;
  const int b = row / a.N;
  const int v0 = part * ACCEPT_PART;
  const bool on = v0 < a.V && a.tokens[(int64_t)b * a.N] >= 0;
  const T* z = (of_draft ? (const T*)a.draft + (int64_t)row * a.ldd : (const T*)a.logits + (int64_t)row * a.ld) + v0;
  float x[16];
  if (on) load_part<T, VEC>(z, min(ACCEPT_PART, a.V - v0), lane, x);
  __syncthreads();
  if (!on) return;
  bool bad = false;
  float m = -CH_INF;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    bad = bad || !(x[i] < CH_INF);
    m = fmaxf(m, x[i]);
  }
  m = wave_max(m);
  double s = 0.0;
  if (m != -CH_INF) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s = s + pow32(exponent(x[i], (double)m, a.scale), table);
  }
  if (bad) s = __builtin_nan("");
  s = wave_sum_f64(s);
  if (lane == 0) {
    const int64_t at = ((int64_t)blockIdx.z * a.B * a.N + row) * a.parts + part;
    a.part_m[at] = m;
    a.part_s[at] = s;
  }
}

// A row's maximum and sum out of its parts, by one wave.  ok: it has a distribution.
struct RowSum {
  double m, s;
  __device__ __forceinline__ bool ok() const { return s > 0.0 && s < HUGE_VAL && m < (double)CH_INF; }
};
__device__ __forceinline__ RowSum row_sum(const AcceptArgs& a, int64_t row, const double* table) {
  const int lane = threadIdx.x & 63;
  const int64_t at = row * a.parts;
  float m = -CH_INF;
  for (int i = lane; i < a.parts; i += 64) m = fmaxf(m, a.part_m[at + i]);
  m = wave_max(m);
  double s = 0.0;
  for (int i = lane; i < a.parts; i += 64) {
    const float pm = a.part_m[at + i];
    const double ps = a.part_s[at + i];
    s = s + (pm == -CH_INF ? ps : ps * pow32(exponent(pm, (double)m, a.scale), table));
  }
  return {(double)m, wave_sum_f64(s)};
}

// ---- the walk ----------------------------------------------------------------------
// Lane u holds node u.  From the root down: a node's children are tested in the order
// of their ids; the walk goes on at the first accepted one and ends where there is
// none.  All rows' sums and all nodes' probabilities come first, so the walk itself
// touches no memory.
struct Walk {
  int node, depth;          // node -1: an empty place
  bool ok;                  // the last row has a distribution
  uint64_t path, rejected;  // nodes on the path; rejected children of the last one
  RowSum p, q;              // of the last row
};
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
  const int tok = lane < a.N ? a.tokens[row0 + lane] : -1;
  const double u = lane < a.N ? a.u[row0 + lane] : 0.0;
  const bool empty = __builtin_amdgcn_readfirstlane(tok) < 0;
  fill_table(sh.table);
  __syncthreads();
  if (!empty)
    for (int i = wave; i < (drawn ? 2 : 1) * a.N; i += WAVES) {
      const int z = i >= a.N ? 1 : 0, r = i - z * a.N;
      const RowSum s = row_sum(a, z * (int64_t)a.B * a.N + row0 + r, sh.table);
      if (lane == 0) sh.rows[z][r] = s;
    }
  __syncthreads();
  if (wave == 0) {
    uint32_t pw = a.tree.parent[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) pw = lane / 4 == i ? a.tree.parent[i] : pw;
    const int parent = lane == 0 ? -1 : (int)(pw >> (8 * (lane & 3))) & 255;
    Walk w{};
    w.node = empty ? -1 : 0;
    if (!empty) {
      const bool named = lane > 0 && lane < a.N && tok >= 0 && tok < a.V;
      double p = 0.0, q = 1.0;
      if (named) {
        const RowSum rp = sh.rows[0][parent];
        p = pow32(exponent(logit<T>((const T*)a.logits + (row0 + parent) * a.ld, tok), rp.m, a.scale), sh.table) / rp.s;
        if (drawn) {
          const RowSum rq = sh.rows[1][parent];
          q = pow32(exponent(logit<T>((const T*)a.draft + (row0 + parent) * a.ldd, tok), rq.m, a.scale), sh.table) / rq.s;
        }
      }
      w.path = 1;
      for (;;) {
        w.rejected = 0;
        w.p = sh.rows[0][w.node];
        w.ok = w.p.ok();
        if (!w.ok) break;
        const uint64_t kids = __ballot(named && parent == w.node);
        if (kids == 0) break;
        if (drawn) {
          w.q = sh.rows[1][w.node];
          w.ok = w.q.ok();
          if (!w.ok) break;
        }
        double left = 1.0;  // the mass of what is not rejected
        int next = -1;
        for (uint64_t rest = kids; rest != 0; rest &= rest - 1) {
          const int c = __ffsll((long long)rest) - 1;
          const double pc = shfl_f64(p, c), uc = shfl_f64(u, c);
          if (uc * (drawn ? shfl_f64(q, c) : left) < pc) {
            next = c;
            break;
          }
          w.rejected |= 1ull << c;
          left = left - pc;
          if (tok == __shfl(tok, c)) p = 0.0;  // a sibling of the same token
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

// Drawn tokens: every part of the residual, grid (groups of four parts, sequences), a
// wave a part.  Each workgroup walks by itself, which is cheaper than a launch between.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void accept_resid_kernel(const AcceptArgs a) {
  __shared__ WalkSpace sh;
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int part = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  accept_walk<T, 4>(a, b, sh);
  const Walk& w = sh.walk;
  const int v0 = part * ACCEPT_PART;
  if (w.node < 0 || !w.ok || w.rejected == 0 || v0 >= a.V) return;
  const int64_t row = (int64_t)b * a.N + w.node;
  const Weights<T> f{(const T*)a.logits + row * a.ld, (const T*)a.draft + row * a.ldd, w.p.m, w.q.m, a.scale,
                     1.0 / w.p.s, 1.0 / w.q.s, sh.table};
  float x[16], xq[16];
  const int n = min(ACCEPT_PART, a.V - v0);
  load_part<T, VEC>(f.z + v0, n, lane, x);
  load_part<T, VEC>(f.zq + v0, n, lane, xq);
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = s + f.of(x[i], xq[i]);
  s = wave_sum_f64(s);
  if (lane == 0) a.resid[(int64_t)b * a.parts + part] = s;
}

// A workgroup of 1024 a sequence: the walk, its results, and the first entry whose
// running sum passes u[0] of the whole, by parts and then within one.
template <typename T, bool VEC>
__global__ __launch_bounds__(1024) void accept_pick_kernel(const AcceptArgs a) {
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row0 = (int64_t)b * a.N;
  const int K1 = a.K + 1;
  __shared__ WalkSpace sh;
  __shared__ int gone[64], n_gone;       // rejected tokens
  __shared__ double wave_s[16], redo[64];
  __shared__ int part_sh, first_sh[16], last_sh[16];
  __shared__ double before_sh, target_sh;
  accept_walk<T, 16>(a, b, sh);
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
    if (tid == 0) a.new_tokens[(int64_t)b * K1 + w.depth] = -1;
    return;
  }
  const int64_t row = row0 + w.node;
  const bool resid = a.draft != nullptr && w.rejected != 0;
  Weights<T> f{(const T*)a.logits + row * a.ld, resid ? (const T*)a.draft + row * a.ldd : nullptr, w.p.m, w.q.m, a.scale,
               resid ? 1.0 / w.p.s : 1.0, resid ? 1.0 / w.q.s : 1.0, sh.table};
  int ng = n_gone;
  auto is_gone = [&](int v) {
    bool g = false;
    for (int i = 0; i < ng; ++i) g = g || gone[i] == v;
    return g;
  };
  // Parts that hold a rejected token are summed without it, a wave each: taking it off
  // the sum would leave rounding where it was most of it.
  for (int i = wave; i < ng; i += 16) {
    const int v0 = gone[i] / ACCEPT_PART * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
    constexpr int E = VEC ? 16 / (int)sizeof(T) : 1;
    float x[16];
    load_part<T, VEC>(f.z + v0, n, lane, x);
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const double one = pow32(exponent(x[k], w.p.m, a.scale), sh.table);
      s = s + (is_gone(v0 + lane * E + 64 * E * (k / E) + k % E) ? 0.0 : one);
    }
    s = wave_sum_f64(s);
    if (lane == 0) redo[i] = s;
  }
  __syncthreads();
  // The part where the running sum passes, by one wave, 64 parts at a time.  Rounding
  // may leave no weight at all behind rejections (the mass that was left was its own
  // error): then the row's own probabilities decide.
  for (int attempt = 0; attempt < 2; ++attempt) {
    if (wave == 0) {
      auto part_weight = [&](int i) {
        if (i >= a.parts) return 0.0;
        if (f.zq != nullptr) return a.resid[(int64_t)b * a.parts + i];
        for (int j = 0; j < ng; ++j)
          if (gone[j] / ACCEPT_PART == i) return redo[j];
        const float pm = a.part_m[row * a.parts + i];
        return pm == -CH_INF ? 0.0 : a.part_s[row * a.parts + i] * pow32(exponent(pm, w.p.m, a.scale), sh.table) * f.one;
      };
      double total = 0.0;
      for (int i0 = 0; i0 < a.parts; i0 += 64) total = total + wave_sum_f64(part_weight(i0 + lane));
      const double u0 = a.u[row0];
      const double target = (u0 > 0.0 ? u0 : 0.0) * total;
      double before = 0.0, last_before = 0.0;
      int last = -1;
      for (int i0 = 0; i0 < a.parts; i0 += 64) {
        const double pw = part_weight(i0 + lane);
        const double upto = before + wave_scan_f64(pw);
        const uint64_t over = __ballot(pw > 0.0 && upto > target), some = __ballot(pw > 0.0);
        const int at = over != 0 ? __ffsll((long long)over) - 1 : some != 0 ? 63 - __clzll((long long)some) : -1;
        if (at >= 0) {
          last = i0 + at;
          last_before = shfl_f64(upto - pw, at);
        }
        if (over != 0) break;
        before = shfl_f64(upto, 63);
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
  if (part_sh < 0) {  // u was no number
    if (tid == 0) a.new_tokens[(int64_t)b * K1 + w.depth] = -1;
    return;
  }
  // within the part, an entry a thread
  static_assert(ACCEPT_PART == 1024, "an entry a thread");
  const int v = part_sh * ACCEPT_PART + tid;
  const double x = v < a.V && !is_gone(v) ? f(v) : 0.0;
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

template <typename T, bool VEC>
void accept_go(const AcceptArgs& a, hipStream_t st) {
  const int groups = (a.parts + 3) / 4;
  hipLaunchKernelGGL((accept_parts_kernel<T, VEC>), dim3(a.B * a.N, groups, a.draft != nullptr ? 2 : 1), dim3(256), 0, st, a);
  if (a.draft != nullptr && a.N > 1)
    hipLaunchKernelGGL((accept_resid_kernel<T, VEC>), dim3(groups, a.B), dim3(256), 0, st, a);
  hipLaunchKernelGGL((accept_pick_kernel<T, VEC>), dim3(a.B), dim3(1024), 0, st, a);
}
template <typename T>
void accept_t(const AcceptArgs& a, hipStream_t st) {
  auto whole = [](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0; };
  if (whole(a.logits, a.ld) && whole(a.draft, a.draft != nullptr ? a.ldd : 0))
    accept_go<T, true>(a, st);
  else
    accept_go<T, false>(a, st);
}

int64_t up(int64_t b) { return (b + 255) / 256 * 256; }

}  // namespace

int64_t accept_bytes(int B, int N, int V, bool drawn) {
  const int64_t parts = (V + ACCEPT_PART - 1) / ACCEPT_PART, rows = (int64_t)B * N * (drawn ? 2 : 1);
  return up(rows * parts * 8) + up(rows * parts * 4) + up(drawn ? B * parts * 8 : 0);
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
}

void launch_accept(int dtype, const AcceptArgs& a, hipStream_t st) {
  if (dtype == DT_BF16)
    accept_t<bf16_t>(a, st);
  else
    accept_t<float>(a, st);
}
