// Rows into a paged K/V cache (paged.h): queries and keys normalised head by head
// and rotated by their position on the way, and the rotation's table.
#include "common.h"
#include "paged.h"

namespace {

// ---- the rotation's table ----------------------------------------------------------
// table[p][i] = gain (cos, sin)(p theta_i), angles in 64 bits and rounded once: at
// position 2^20 a 32-bit angle is off by up to 0.06.  A thread an entry; bound by the
// 64-bit power, sine and cosine: 33024 positions of 64 pairs take 27 us, once a model.
__global__ __launch_bounds__(256) void rope_table_kernel(const RopeArgs r, float2* __restrict__ table, int64_t n) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (e >= n) return;
  const int64_t p = e / r.pairs;
  const int i = (int)(e - p * r.pairs);
  double th = pow((double)r.base, -(double)(2 * i) / (double)(2 * r.pairs));
  if (r.scaling == 1) {
    th = th / (double)r.factor;
  } else if (r.scaling == 2) {
    // turns that the original context holds: many keep theta, few divide it
    const double t = (double)r.original * th / 6.283185307179586476925;
    const double w = fmin(fmax((t - (double)r.low) / ((double)r.high - (double)r.low), 0.0), 1.0);
    th = th * (w + (1.0 - w) / (double)r.factor);
  }
  double s, c;
  sincos((double)p * th, &s, &c);
  table[e] = float2{(float)(c * (double)r.gain), (float)(s * (double)r.gain)};
}

// ---- rows --------------------------------------------------------------------------
// Four values at any element: 16 (8) bytes at once.
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void load4(const float* p, float* x) {
  const f4_any v = *reinterpret_cast<const f4_any*>(p);
  x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
}
__device__ __forceinline__ void load4(const bf16_t* p, float* x) {
  const u2_any v = *reinterpret_cast<const u2_any*>(p);
  x[0] = __uint_as_float(v.x << 16), x[1] = __uint_as_float(v.x & 0xffff0000u);
  x[2] = __uint_as_float(v.y << 16), x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float* x) {
  *reinterpret_cast<f4_any*>(p) = f4_any{x[0], x[1], x[2], x[3]};
}
__device__ __forceinline__ void store4(bf16_t* p, const float* x) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  *reinterpret_cast<u2_any*>(p) = u2_any{__builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x[0], x[1]}, b2)),
                                       __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x[2], x[3]}, b2))};
}

// HD / 8 lanes a head, eight values a lane: four pairs of the rotation, so nothing
// but the norm's sum crosses lanes.  Pairs (i, i + P): values 4 j .. and P + 4 j ..
// of lane j, the ones past the rotated part in order after them.  Neighbouring
// pairs: eight values in a row.  VEC: both are runs of four values (P a multiple of
// 4); else a value at a time.
// Bound by the bytes of many rows and by the launch of few: 2044 32-bit rows of 48 heads
// into bf16 (76 MB) 17.6 us, 4.35 TB/s; one row 2.9 us, eight normed rows 3.3.
// Elements of value v (0 .. 7) of lane j: pair v / 2 in either layout.
__device__ __forceinline__ int element(int j, int v, int P, bool cross) {
  const int u = 4 * j + (v >> 1);
  return cross && u < P ? u + (v & 1) * P : 2 * u + (v & 1);
}

// x[2 i], x[2 i + 1]: pair i of the lane.
template <typename T, bool VEC>
__device__ __forceinline__ void load_pairs(const T* p, int j, int P, bool cross, float* x) {
  if constexpr (VEC) {
    const bool turned = cross && 4 * j < P;
    float a[8];
    load4(p + (turned ? 4 * j : 8 * j), a);
    load4(p + (turned ? P + 4 * j : 8 * j + 4), a + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = turned ? a[i] : a[2 * i];
      x[2 * i + 1] = turned ? a[4 + i] : a[2 * i + 1];
    }
  } else {
#pragma unroll
    for (int v = 0; v < 8; ++v) x[v] = ET<T>::to_f(p[element(j, v, P, cross)]);
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_pairs(T* p, int j, int P, bool cross, const float* x) {
  if constexpr (VEC) {
    const bool turned = cross && 4 * j < P;
    float a[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = turned ? x[2 * i] : x[i];
      a[4 + i] = turned ? x[2 * i + 1] : x[4 + i];
    }
    store4(p + (turned ? 4 * j : 8 * j), a);
    store4(p + (turned ? P + 4 * j : 8 * j + 4), a + 4);
  } else {
#pragma unroll
    for (int v = 0; v < 8; ++v) p[element(j, v, P, cross)] = ET<T>::from_f(x[v]);
  }
}

template <int HD>
__device__ __forceinline__ float head_sum(float v) {  // over the HD / 8 lanes of a head
  if constexpr (HD == 128) return row16_sum(v);
  v = v + dpp_mov<DPP_XOR1>(v);
  v = v + dpp_mov<DPP_XOR2>(v);
  return v + dpp_mov<DPP_MIRROR8>(v);
}

// y = x (mean(x^2) + eps)^-1/2 gain.  Where mean + eps is not between 2^-100 and 2^128 it
// is formed again of values scaled by k, a power of two: by 2^60, which leaves no square
// that counts below the normal numbers, or by 2^-68, so that 128 squares of the largest float
// stay below 2^127.  An infinity makes its own value NaN and the others 0, as the formula
// does.
template <int HD>
__device__ __forceinline__ void head_norm(float (&x)[8], const float (&gain)[8], float eps) {
  float ss = 0.f;
#pragma unroll
  for (int v = 0; v < 8; ++v) ss = fmaf(x[v], x[v], ss);
  float t = head_sum<HD>(ss) * (1.0f / HD) + eps, back = 1.f;
  const bool low = t < 0x1p-100f, high = t == CH_INF;
  if (__ballot(low || high) != 0) {
    const float k = low ? 0x1p60f : high ? 0x1p-68f : 1.f;
    float s2 = 0.f;
#pragma unroll
    for (int v = 0; v < 8; ++v) s2 = fmaf(x[v] * k, x[v] * k, s2);
    t = head_sum<HD>(s2) * (1.0f / HD) + eps * k * k;
    // small values are scaled before their product, which might lose bits, large ones after
#pragma unroll
    for (int v = 0; v < 8; ++v) x[v] = low ? x[v] * k : x[v];
    back = low ? 1.f : k;
  }
  const float r = 1.0f / sqrtf(t);
#pragma unroll
  for (int v = 0; v < 8; ++v) x[v] = x[v] * r * back * gain[v];
}

// Grid (blocks of a row's heads, rows).  A lane does the same eight places of
// every head it takes, so the table and the gains are read once.
template <typename TI, typename TC, int HD, bool VEC>
__global__ __launch_bounds__(256) void paged_append_kernel(const PagedView c, const AppendArgs a) {
  constexpr int L = HD / 8, PER = 256 / L;
  const int j = threadIdx.x % L, slot = blockIdx.x * PER + threadIdx.x / L;
  const int P = a.pairs;
  const bool cross = a.cross != 0;
  const int heads = a.Hq + 2 * c.H;
  for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const int b = a.seq[row], p = a.pos[row];
    if (b < 0 || b >= c.B || (P > 0 && p >= a.positions)) continue;
    const uint32_t base = paged_row(c, c.page_table + (int64_t)b * c.max_pages, p);
    if (base == PAGED_NONE) continue;
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cs[i] = 1.f, sn[i] = 0.f;
      if (4 * j + i < P) {
        const float2 t = a.table[(int64_t)p * P + 4 * j + i];
        cs[i] = t.x, sn[i] = t.y;
      }
    }
    for (int h = slot; h < heads; h += PER * gridDim.x) {  // the lanes of a head stay together
      const bool is_q = h < a.Hq, is_v = h >= a.Hq + c.H;
      const int kvh = h - a.Hq - (is_v ? c.H : 0);
      const TI* src = is_q ? (const TI*)a.q + row * a.ld + h * HD
                           : (const TI*)(is_v ? a.v : a.k) + row * a.ld + kvh * HD;
      float x[8];
      load_pairs<TI, VEC>(src, j, P, cross, x);
      if (!is_v) {
        const float* gain = is_q ? a.q_gain : a.k_gain;
        if (gain != nullptr) {
          float g[8];
          load_pairs<float, VEC>(gain, j, P, cross, g);
          head_norm<HD>(x, g, a.eps);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * j + i < P) {
            const float u = x[2 * i], w = x[2 * i + 1];
            x[2 * i] = u * cs[i] - w * sn[i];
            x[2 * i + 1] = u * sn[i] + w * cs[i];
          }
      }
      TC* dst = is_q ? (TC*)a.q_out + row * a.ldo + h * HD
                     : (TC*)c.pool + ((uint64_t)base + (uint64_t)((is_v ? c.H : 0) + kvh) * c.ps.d) * HD;
      store_pairs<TC, VEC>(dst, j, P, cross, x);
    }
  }
}

template <typename TI, typename TC, int HD>
void append_go(const PagedView& c, const AppendArgs& a, bool vec, hipStream_t st) {
  constexpr int PER = 256 / (HD / 8);
  const int heads = a.Hq + 2 * c.H;
  const dim3 grid((heads + PER - 1) / PER, a.rows < 65535 ? a.rows : 65535);
  if (vec)
    hipLaunchKernelGGL((paged_append_kernel<TI, TC, HD, true>), grid, dim3(256), 0, st, c, a);
  else
    hipLaunchKernelGGL((paged_append_kernel<TI, TC, HD, false>), grid, dim3(256), 0, st, c, a);
}
template <typename TI, typename TC>
void append_t(const PagedView& c, const AppendArgs& a, bool vec, hipStream_t st) {
  if (c.hd == 128)
    append_go<TI, TC, 128>(c, a, vec, st);
  else
    append_go<TI, TC, 64>(c, a, vec, st);
}

}  // namespace

void launch_rope_table(const RopeArgs& r, void* table, int positions, hipStream_t st) {
  const int64_t n = (int64_t)positions * r.pairs;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, r, (float2*)table, n);
}

void launch_paged_append(int dtype, int held, const PagedView& c, const AppendArgs& a, hipStream_t st) {
  const bool vec = a.cross == 0 || a.pairs % 4 == 0;
  if (dtype == DT_BF16)
    held == DT_BF16 ? append_t<bf16_t, bf16_t>(c, a, vec, st) : append_t<bf16_t, float>(c, a, vec, st);
  else
    held == DT_BF16 ? append_t<float, bf16_t>(c, a, vec, st) : append_t<float, float>(c, a, vec, st);
}
