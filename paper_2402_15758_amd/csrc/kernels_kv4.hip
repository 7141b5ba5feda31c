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

// Attention, one wave per (sequence, node, head): a lane scores one key of 64,
// then owns head_dim / 64 output dimensions over them.
template <typename T, int HD>
__global__ __launch_bounds__(64) void kv4_attn_kernel(const Kv4AttnArgs a) {
  constexpr int DPL = HD / 64;
  const Kv4View& c = a.c;
  const int h = blockIdx.x, u = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
  const int hk = h / (a.Hq / c.H);
  const int64_t row = (int64_t)b * a.N + u;
  const int n = min(a.n_b[b], c.max_pages * c.ps);  // what lies past the table is not seen anyway
  T* out = (T*)a.out + row * a.ldo + h * HD + DPL * lane;
  const T* qrow = (const T*)a.q + row * a.ldq + h * HD;
  const int total = n < 0 ? 0 : n + a.tree.depth[u] + 1;
  float m = -CH_INF, l = 0.f, o[DPL];
#pragma unroll
  for (int d = 0; d < DPL; ++d) o[d] = 0.f;
  for (int k0 = 0; k0 < total; k0 += 64) {
    const int key = k0 + lane;
    const int p = key < n ? key : n + a.tree.path[u][min(key - n, KV4_MAX_DEPTH)];
    int64_t e = key < total ? kv4_slot(c, b, p) : -1;
    if (e >= 0) e += (int64_t)hk * c.ps * HD;
    float s = 0.f;
    if (e >= 0) {
      for (int g = 0; g < HD / 32; ++g) {
        const float sc = fp4_scale(c.scales[e / 32 + g]);
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(c.codes + e / 2 + g * 16 + 4 * j);
          const f32x4 x = fp4_to_f32x4<0>(w, sc), y = fp4_to_f32x4<1>(w, sc);
          for (int t = 0; t < 4; ++t) s = fmaf(ET<T>::to_f(qrow[g * 32 + 8 * j + t]), x[t], s);
          for (int t = 0; t < 4; ++t) s = fmaf(ET<T>::to_f(qrow[g * 32 + 8 * j + 4 + t]), y[t], s);
        }
      }
    }
    s = e >= 0 ? s * (a.scale * LOG2E) : -CH_INF;
    if (__ballot(e >= 0) == 0) continue;
    const float mn = fmaxf(m, wave_max(s));
    const float alpha = m == -CH_INF ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    const float pe = e >= 0 ? __builtin_amdgcn_exp2f(s - mn) : 0.f;
    l = l * alpha + wave_sum(pe);
    m = mn;
#pragma unroll
    for (int d = 0; d < DPL; ++d) o[d] *= alpha;
    for (int j = 0; j < 64; ++j) {
      const int64_t ej = __shfl((long long)e, j);
      const float pj = __shfl(pe, j);
      if (ej < 0) continue;
      const int64_t ve = ej + (int64_t)c.H * c.ps * HD + DPL * lane;
      const float sc = fp4_scale(c.scales[ve / 32]);
      const uint32_t w = (uint32_t)c.codes[ve / 2] >> (DPL == 1 ? 4 * (lane & 1) : 0);
      const f32x4 x = fp4_to_f32x4<0>(w, sc);
#pragma unroll
      for (int d = 0; d < DPL; ++d) o[d] = fmaf(pj, x[d], o[d]);
    }
  }
#pragma unroll
  for (int d = 0; d < DPL; ++d) out[d] = ET<T>::from_f(l == 0.f ? 0.f : o[d] / l);
}

template <typename T, int HD>
void kv4_attn_go(const Kv4AttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((kv4_attn_kernel<T, HD>), dim3(a.Hq, a.N, a.c.B), dim3(64), 0, st, a);
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

int64_t kv4_attn_bytes(int, int64_t, int, int, int) { return 256; }

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
