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

// e^x for x <= 0 (or NaN), relative error below 2^-50: x = n ln 2 + r, |r| <= ln 2 / 2,
// with ln 2 in two parts, and Taylor's series of e^r up to r^12 / 12! (the next term is
// below 2^-52 / 8).  0 from -745.2 on.
__device__ __forceinline__ double exp_neg(double x) {
  const double y = fmax(x, -800.0);
  const double n = rint(y * 1.4426950408889634074);
  double r = fma(n, -0x1.62e42fee00000p-1, y);
  r = fma(n, -0x1.a39ef35793c76p-33, r);
  double p = 1.0 / 479001600.0;
  p = fma(p, r, 1.0 / 39916800.0);
  p = fma(p, r, 1.0 / 3628800.0);
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

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

// ---- parts of rows -----------------------------------------------------------------
// Grid (rows, parts, target | draft).  A thread holds its entries, so a row is read
// once.  A NaN or +inf makes the part's sum NaN: such a row has no distribution.
template <typename T>
__global__ __launch_bounds__(256) void accept_parts_kernel(const AcceptArgs a) {
  constexpr int E = ACCEPT_PART / 256;
  const int part = blockIdx.y, row = blockIdx.x, tid = threadIdx.x;
  const bool of_draft = blockIdx.z != 0;
  const int b = row / a.N;
  if (a.tokens[(int64_t)b * a.N] < 0) return;  // an empty place
  const void* z = of_draft ? (const void*)((const T*)a.draft + (int64_t)row * a.ldd)
                           : (const void*)((const T*)a.logits + (int64_t)row * a.ld);
  const int v0 = part * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
  float x[E];
  bool bad = false;
  float m = -CH_INF;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int v = tid + 256 * i;
    x[i] = v < n ? logit<T>(z, v0 + v) : -CH_INF;
    bad = bad || !(x[i] < CH_INF);
    m = fmaxf(m, x[i]);
  }
  __shared__ float msh[4];
  __shared__ double ssh[4];
  m = wave_max(m);
  if ((tid & 63) == 0) msh[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(msh[0], msh[1]), fmaxf(msh[2], msh[3]));
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < E; ++i)
    s = s + (x[i] == -CH_INF ? 0.0 : exp_neg(((double)x[i] - (double)m) * a.inv_T));
  if (bad) s = __builtin_nan("");
  s = wave_sum_f64(s);
  if ((tid & 63) == 0) ssh[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    const int64_t at = ((int64_t)blockIdx.z * a.B * a.N + row) * a.parts + part;
    a.part_m[at] = m;
    a.part_s[at] = (ssh[0] + ssh[1]) + (ssh[2] + ssh[3]);
  }
}

// A row's maximum and sum out of its parts, by one wave.  ok: it has a distribution.
struct RowSum {
  double m, s;
  bool ok;
};
__device__ __forceinline__ RowSum row_sum(const AcceptArgs& a, int64_t row, bool of_draft) {
  const int lane = threadIdx.x & 63;
  const int64_t at = ((of_draft ? (int64_t)a.B * a.N : 0) + row) * a.parts;
  float m = -CH_INF;
  for (int i = lane; i < a.parts; i += 64) m = fmaxf(m, a.part_m[at + i]);
  m = wave_max(m);
  double s = 0.0;
  for (int i = lane; i < a.parts; i += 64) {
    const float pm = a.part_m[at + i];
    const double ps = a.part_s[at + i];
    s = s + (pm == -CH_INF ? ps : ps * exp_neg(((double)pm - (double)m) * a.inv_T));
  }
  s = wave_sum_f64(s);
  return {(double)m, s, s > 0.0 && s < HUGE_VAL && m < CH_INF};
}

// ---- the walk ----------------------------------------------------------------------
// Lane u holds node u.  From the root down: a node's children are tested in the order
// of their ids; the walk goes on at the first accepted one and ends where there is
// none.  One wave; the result is uniform.
struct Walk {
  int node, depth;          // node -1: an empty place
  bool ok;                  // the last row has a distribution
  uint64_t path, rejected;  // nodes on the path; rejected children of the last one
  RowSum p, q;              // of the last row
};
template <typename T>
__device__ Walk accept_walk(const AcceptArgs& a, int b) {
  const int lane = threadIdx.x & 63;
  uint32_t pw = a.tree.parent[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) pw = lane / 4 == i ? a.tree.parent[i] : pw;
  const int parent = lane == 0 ? -1 : (int)(pw >> (8 * (lane & 3))) & 255;
  const int64_t row0 = (int64_t)b * a.N;
  const int tok = lane < a.N ? a.tokens[row0 + lane] : -1;
  const double u = lane < a.N ? a.u[row0 + lane] : 0.0;
  Walk w{};
  if (__builtin_amdgcn_readfirstlane(tok) < 0) {
    w.node = -1;
    return w;
  }
  const bool named = lane > 0 && lane < a.N && tok >= 0 && tok < a.V;
  w.path = 1;
  for (;;) {
    w.rejected = 0;
    w.p = row_sum(a, row0 + w.node, false);
    w.ok = w.p.ok;
    if (!w.ok) return w;
    uint64_t kids = __ballot(named && parent == w.node);
    if (kids == 0) return w;
    if (a.draft != nullptr) {
      w.q = row_sum(a, row0 + w.node, true);
      w.ok = w.q.ok;
      if (!w.ok) return w;
    }
    double p = 0.0, q = 1.0;
    if ((kids >> lane) & 1) {
      const double z = (double)logit<T>((const T*)a.logits + (row0 + w.node) * a.ld, tok);
      p = exp_neg((z - w.p.m) * a.inv_T) / w.p.s;
      if (a.draft != nullptr) {
        const double zq = (double)logit<T>((const T*)a.draft + (row0 + w.node) * a.ldd, tok);
        q = exp_neg((zq - w.q.m) * a.inv_T) / w.q.s;
      }
    }
    double left = 1.0;  // the mass of what is not rejected
    int next = -1;
    for (uint64_t rest = kids; rest != 0; rest &= rest - 1) {
      const int c = __ffsll((long long)rest) - 1;
      const double pc = shfl_f64(p, c), uc = shfl_f64(u, c);
      if (uc * (a.draft != nullptr ? shfl_f64(q, c) : left) < pc) {
        next = c;
        break;
      }
      w.rejected |= 1ull << c;
      left = left - pc;
      if (tok == __shfl(tok, c)) p = 0.0;  // a sibling of the same token
    }
    if (next < 0) return w;
    w.node = next;
    w.depth += 1;
    w.path |= 1ull << next;
  }
}

// ---- the next token ------------------------------------------------------------------
// Weight of entry v where a walk ended: the target's probability (times the row's sum)
// where it is not a rejected token, or what the draft leaves of it.
template <typename T>
struct Weights {
  const T *z, *zq;          // zq: nullptr without a residual
  double m, mq, inv_T, scale, scale_q;
  __device__ __forceinline__ double operator()(int v) const {
    const double p = exp_neg(((double)ET<T>::to_f(z[v]) - m) * inv_T) * scale;
    if (zq == nullptr) return p;
    return fmax(p - exp_neg(((double)ET<T>::to_f(zq[v]) - mq) * inv_T) * scale_q, 0.0);
  }
};

// Drawn tokens: every part of the residual, grid (parts, sequences).  Each workgroup
// walks by itself, which is cheaper than a launch between.
template <typename T>
__global__ __launch_bounds__(256) void accept_resid_kernel(const AcceptArgs a) {
  const int part = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  __shared__ Walk wsh;
  if (tid < 64) {
    const Walk w = accept_walk<T>(a, b);
    if (tid == 0) wsh = w;
  }
  __syncthreads();
  const Walk w = wsh;
  if (w.node < 0 || !w.ok || w.rejected == 0) return;
  const int64_t row = (int64_t)b * a.N + w.node;
  const Weights<T> f{(const T*)a.logits + row * a.ld, (const T*)a.draft + row * a.ldd, w.p.m, w.q.m, a.inv_T,
                     1.0 / w.p.s, 1.0 / w.q.s};
  const int v0 = part * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
  double s = 0.0;
  for (int v = tid; v < n; v += 256) s = s + f(v0 + v);
  s = wave_sum_f64(s);
  __shared__ double ssh[4];
  if ((tid & 63) == 0) ssh[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) a.resid[(int64_t)b * a.parts + part] = (ssh[0] + ssh[1]) + (ssh[2] + ssh[3]);
}

// A workgroup of 1024 a sequence: the walk, its results, and the first entry whose
// running sum passes u[0] of the whole, by parts and then within one.
template <typename T>
__global__ __launch_bounds__(1024) void accept_pick_kernel(const AcceptArgs a) {
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row0 = (int64_t)b * a.N;
  const int K1 = a.K + 1;
  __shared__ Walk wsh;
  __shared__ int gone[64], n_gone;       // rejected tokens
  __shared__ double wave_s[16], redo[64];
  __shared__ int part_sh;
  __shared__ double before_sh, target_sh;
  if (tid < 64) {
    const Walk w = accept_walk<T>(a, b);
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
      wsh = w;
      part_sh = -1;
      n_gone = a.draft == nullptr ? __popcll(w.rejected) : 0;
    }
    if (a.draft == nullptr && ((w.rejected >> lane) & 1)) gone[__popcll(w.rejected & ((1ull << lane) - 1))] = tok;
  }
  __syncthreads();
  const Walk w = wsh;
  if (w.node < 0) return;
  if (!w.ok) {
    if (tid == 0) a.new_tokens[(int64_t)b * K1 + w.depth] = -1;
    return;
  }
  const int64_t row = row0 + w.node;
  const bool resid = a.draft != nullptr && w.rejected != 0;
  Weights<T> f{(const T*)a.logits + row * a.ld, resid ? (const T*)a.draft + row * a.ldd : nullptr, w.p.m, w.q.m, a.inv_T,
               resid ? 1.0 / w.p.s : 1.0, resid ? 1.0 / w.q.s : 1.0};
  int ng = n_gone;
  auto weight_of = [&](int v) {
    for (int i = 0; i < ng; ++i)
      if (gone[i] == v) return 0.0;
    return f(v);
  };
  // parts that hold a rejected token are summed without it, a wave each: taking it off
  // the sum would leave rounding where it was most of it
  for (int i = wave; i < ng; i += 16) {
    const int v0 = gone[i] / ACCEPT_PART * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
    double s = 0.0;
    for (int v = lane; v < n; v += 64) s = s + weight_of(v0 + v);
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
        return pm == -CH_INF ? 0.0 : a.part_s[row * a.parts + i] * exp_neg(((double)pm - w.p.m) * a.inv_T);
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
    f.scale = 1.0;
  }
  if (part_sh < 0) {  // u was no number
    if (tid == 0) a.new_tokens[(int64_t)b * K1 + w.depth] = -1;
    return;
  }
  // within the part: four entries a thread, in order
  const int v0 = part_sh * ACCEPT_PART, n = min(ACCEPT_PART, a.V - v0);
  double x[4], s = 0.0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = 4 * tid + i < n ? weight_of(v0 + 4 * tid + i) : 0.0;
    s = s + x[i];
  }
  const double scan = wave_scan_f64(s);
  if (lane == 63) wave_s[wave] = scan;
  __syncthreads();
  double run = before_sh;
  for (int i = 0; i < wave; ++i) run = run + wave_s[i];
  run = run + (scan - s);
  int mine = 0x7fffffff, pos = -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    run = run + x[i];
    if (x[i] > 0.0) {
      if (run > target_sh && mine == 0x7fffffff) mine = v0 + 4 * tid + i;
      pos = v0 + 4 * tid + i;
    }
  }
  // the first that passes; where rounding leaves none, the last with any weight
  __shared__ int first_sh[16], last_sh[16];
  const int wf = wave_min_i(mine), wl = -wave_min_i(-pos);
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

template <typename T>
void accept_t(const AcceptArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((accept_parts_kernel<T>), dim3(a.B * a.N, a.parts, a.draft != nullptr ? 2 : 1), dim3(256), 0, st,
                     a);
  if (a.draft != nullptr && a.N > 1)
    hipLaunchKernelGGL((accept_resid_kernel<T>), dim3(a.parts, a.B), dim3(256), 0, st, a);
  hipLaunchKernelGGL((accept_pick_kernel<T>), dim3(a.B), dim3(1024), 0, st, a);
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
