// Products with 4-bit weights: Y = X[M][K] @ W[K][N], W in groups of 32 along
// the reduction (fp4.h).  A weight is converted to the activations' type in
// registers (exactly) and enters the same MFMAs, in the same order, as the bf16
// weights of kernels_gemm.hip: per reduction slice four sums, one per residue
// class of the k-blocks mod 4, added in class order, then the slices in slice
// order.  So a bf16 product has the bits of the bf16 kernels' product with the
// converted matrix, whatever its row count, and launches of many rows may take
// that route (gemm_fp4_unpacks).
//
// Layout (a quarter of the bf16 bytes plus 1/16 of that for scales): unit
// (column block c, slice s, class w, quad q) holds four successive k-blocks of
// the class, kb = kps s + w + 4 (4 q + i).  Lane l's 16 bytes are the words of
// k-blocks i = 0..3, each with k = 32 kb + 8 (l >> 4) + 0..7 of column 16 c +
// (l & 15): 1 KiB contiguous a load.  Its scales are 64 bytes, four (i) a column.
#include <hip/hip_ext.h>

#include <algorithm>

#include "common.h"
#include "fp4.h"
#include "gemm_epilogue.h"
#include "kernels.h"

namespace {

// Where the units of a packed matrix lie.
struct Fp4Shape {
  int N, K, splits, kps, quads;  // quads: units per class and slice
  int64_t codes_bytes;
};
__host__ __device__ inline Fp4Shape fp4_shape(int N, int K, int splits) {
  Fp4Shape s;
  s.N = N;
  s.K = K;
  s.splits = splits;
  s.kps = K / FP4_GROUP / splits;
  s.quads = ((s.kps + 3) / 4 + 3) / 4;
  s.codes_bytes = (int64_t)(N / 16) * splits * 4 * s.quads * 1024;
  return s;
}
__device__ __forceinline__ int64_t fp4_unit(const Fp4Shape& s, int c, int slice, int cls) {
  return (((int64_t)c * s.splits + slice) * 4 + cls) * s.quads;
}

// Column of packed block c, lane column cl (the packings of kernels_gemm.hip).
struct Fp4Src {
  int which, col;
};
__device__ __forceinline__ Fp4Src fp4_source(int kind, int c, int cl, int H, int hd) {
  if (kind == PACK_QKV) {
    const int per_sec = H * hd / 16, sec = c / per_sec, within = c % per_sec;
    const int h = within / (hd / 16), q = within % (hd / 16);
    const int dim = sec < 2 ? (cl < 8 ? 8 * q + cl : hd / 2 + 8 * q + cl - 8) : 16 * q + cl;
    return {sec, h * hd + dim};
  }
  if (kind == PACK_GU) return {cl < 8 ? 0 : 1, 8 * c + (cl & 7)};
  return {0, 16 * c + cl};
}

// One wave a unit; a group's 32 values lie in the four lanes of a column.
template <typename T>
__global__ __launch_bounds__(256) void fp4_pack_kernel(const T* __restrict__ s0, const T* __restrict__ s1,
                                                       const T* __restrict__ s2, int64_t ldw, int kind, int H, int hd,
                                                       const Fp4Shape sh, uint8_t* __restrict__ dst) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= sh.codes_bytes / 1024) return;  // whole waves
  const int lane = threadIdx.x & 63;
  const int quad = (int)(unit % sh.quads), cls = (int)(unit / sh.quads % 4);
  const int slice = (int)(unit / sh.quads / 4 % sh.splits), c = (int)(unit / sh.quads / 4 / sh.splits);
  const Fp4Src src = fp4_source(kind, c, lane & 15, H, hd);
  const T* base = (src.which == 0 ? s0 : (src.which == 1 ? s1 : s2)) + src.col;
  uint32_t w[4], sc = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int in_slice = cls + 4 * (4 * quad + i);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (in_slice < sh.kps) {
      const int64_t k0 = (int64_t)(slice * sh.kps + in_slice) * FP4_GROUP + (lane >> 4) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = ET<T>::to_f(base[(k0 + e) * ldw]);
    }
    uint32_t m = amax_bits8(v);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    const uint32_t s = fp4_scale_byte(m);
    w[i] = fp4_encode8(v, s);
    sc |= s << (8 * i);
  }
  st16(dst + unit * 1024 + lane * 16, int4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]});
  if (lane < 16) reinterpret_cast<uint32_t*>(dst + sh.codes_bytes + unit * 64)[lane] = sc;
}

// The values: row-major [K][N] (ROWS), or bf16 in the layout of the bf16
// kernels (kernels_gemm.hip), N rounded up to whole 64-column groups.
template <typename T, bool ROWS>
__global__ __launch_bounds__(256) void fp4_unpack_kernel(const uint8_t* __restrict__ src, const Fp4Shape sh,
                                                         T* __restrict__ dst, int64_t ldw) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= sh.codes_bytes / 1024) return;
  const int lane = threadIdx.x & 63;
  const int quad = (int)(unit % sh.quads), cls = (int)(unit / sh.quads % 4);
  const int slice = (int)(unit / sh.quads / 4 % sh.splits), c = (int)(unit / sh.quads / 4 / sh.splits);
  const int4 code = ld16(src + unit * 1024 + lane * 16);
  const uint32_t sc = reinterpret_cast<const uint32_t*>(src + sh.codes_bytes + unit * 64)[lane & 15];
  const int kblocks = sh.K / FP4_GROUP;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int in_slice = cls + 4 * (4 * quad + i);
    if (in_slice >= sh.kps) break;  // wave-uniform
    const int kb = slice * sh.kps + in_slice;
    const uint32_t w = (uint32_t)(i == 0 ? code.x : (i == 1 ? code.y : (i == 2 ? code.z : code.w)));
    const float s = fp4_scale((sc >> (8 * i)) & 255);
    if constexpr (ROWS) {
      const f32x4 a = fp4_to_f32x4<0>(w, s), b = fp4_to_f32x4<1>(w, s);
      T* d = dst + ((int64_t)kb * FP4_GROUP + (lane >> 4) * 8) * ldw + 16 * c + (lane & 15);
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e * ldw] = ET<T>::from_f(e < 4 ? a[e & 3] : b[e & 3]);
    } else {
      st16(dst + ((((int64_t)(c / NB) * kblocks + kb) * NB + c % NB) * 64 + lane) * 8, fp4_to_bf16x8(w, s));
    }
  }
}

// X rows of a launch: tiled (fragment order, x_mtiles 16-row tiles) or row-major
// with a row stride (up to 16 rows: M == 1 reads 64 bytes a k-block).
template <typename T, bool RM>
struct XRows {
  const T* base;
  int64_t step;   // elements from one 32-wide k-block to the next
  int64_t tile;   // from one 16-row tile to the next
  int64_t half;   // fp32: from the first four indices of a lane to the next four
  __device__ __forceinline__ XRows(const GemmShape& sh, int64_t ldx, int mb0, int lane) {
    const int g = lane >> 4, r = lane & 15;
    if constexpr (RM) {  // rows past M repeat the last one; they are not stored
      base = (const T*)sh.X + (int64_t)min(r, sh.M - 1) * ldx + 8 * g;
      step = 32;
      tile = 0;
      half = 4;
    } else if constexpr (sizeof(T) == 2) {
      base = (const T*)sh.X + ((int64_t)mb0 * 64 + lane) * 8;
      step = (int64_t)sh.x_mtiles * 64 * 8;
      tile = 64 * 8;
      half = 0;
    } else {  // two fp32 k-blocks of 16: lanes of pieces 2 (g & 1) and 2 (g & 1) + 1 of block g >> 1
      base = (const T*)sh.X + (((int64_t)(g >> 1) * sh.x_mtiles + mb0) * 64 + 32 * (g & 1) + r) * 4;
      step = (int64_t)sh.x_mtiles * 64 * 8;
      tile = 64 * 4;
      half = 16 * 4;
    }
  }
  __device__ __forceinline__ void load(int kb, int i, Frag32<T>& f) const {
    const T* p = base + (int64_t)kb * step + i * tile;
    f.v[0] = ld16(p);
    if constexpr (sizeof(T) == 4) f.v[1] = ld16(p + half);
  }
};

__device__ __forceinline__ int4 ld16_nt(const void* p) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 v = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p));
  return int4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ uint32_t word(const int4& v, int i) {
  return (uint32_t)(i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)));
}

// One workgroup's run of CB column blocks from cb0, rows 16 mb0 .. 16 (mb0 +
// MB) - 1 of one slice; the four waves take one class each.
template <typename T, int MB, int CB, bool RM>
__device__ __forceinline__ void fp4_run(const GemmShape& sh, const GemmEpi& e, int64_t ldx, const Fp4Shape& w4,
                                        int kind, int cb0, int mb0, int slice, f32x4* red, const RowMeta* rm,
                                        float* stage) {
  constexpr int XP = MB >= 4 ? 2 : 4;  // k-blocks of X in flight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint8_t* codes[CB];
  const uint8_t* scales[CB];
#pragma unroll
  for (int j = 0; j < CB; ++j) {
    const int64_t u = fp4_unit(w4, cb0 + j, slice, wave);
    codes[j] = (const uint8_t*)sh.W + u * 1024 + lane * 16;
    scales[j] = (const uint8_t*)sh.W + w4.codes_bytes + u * 64 + (lane & 15) * 4;
  }
  const XRows<T, RM> X(sh, ldx, mb0, lane);
  const int kfirst = slice * w4.kps + wave;
  const int nk = wave < w4.kps ? (w4.kps - wave + 3) / 4 : 0;  // k-blocks of this wave
  const int nq = (nk + 3) / 4;

  f32x4 acc[MB][CB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < CB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  int4 bc[2][CB];
  uint32_t bs[2][CB];
  Frag32<T> bx[XP][MB];
  auto load_w = [&](int slot, int q) {
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      bc[slot][j] = ld16_nt(codes[j] + (int64_t)q * 1024);
      bs[slot][j] = *reinterpret_cast<const uint32_t*>(scales[j] + (int64_t)q * 64);
    }
  };
  auto load_x = [&](int slot, int t) {  // past the last k-block: the last again
#pragma unroll
    for (int i = 0; i < MB; ++i) X.load(kfirst + 4 * min(t, nk - 1), i, bx[slot][i]);
  };
  auto block = [&](int slot, int i, int xs) {
#pragma unroll
    for (int j = 0; j < CB; ++j) {
      Frag32<T> w;
      w.from_fp4(word(bc[slot][j], i), fp4_scale((bs[slot][j] >> (8 * i)) & 255));
#pragma unroll
      for (int r = 0; r < MB; ++r) acc[r][j] = mfma32<T>(bx[xs][r], w, acc[r][j]);
    }
  };
  if (nk > 0) {
    load_w(0, 0);
#pragma unroll
    for (int t = 0; t < XP; ++t) load_x(t, t);
    int q = 0;
    for (; q + 2 < nq; q += 2) {  // both quads whole
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load_w(1 - h, q + h + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          block(h, i, i % XP);
          load_x(i % XP, 4 * (q + h) + i + XP);
        }
      }
    }
    // one or two quads left, the last of them perhaps cut short
    if (q + 2 == nq) {
      load_w(1, q + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        block(0, i, i % XP);
        load_x(i % XP, 4 * q + i + XP);
      }
      ++q;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (4 * q + i < nk) {  // wave-uniform
          block(1, i, i % XP);
          load_x(i % XP, 4 * q + i + XP);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (4 * q + i < nk) {
          block(0, i, i % XP);
          load_x(i % XP, 4 * q + i + XP);
        }
      }
    }
  }

  // the classes meet in LDS, in class order
  constexpr int JR = CB < 32 / MB ? CB : 32 / MB;
#pragma unroll
  for (int j0 = 0; j0 < CB; j0 += JR) {
    if (j0 > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int jj = 0; jj < JR; ++jj)
        if (j0 + jj < CB) red[((wave * MB + i) * JR + jj) * 64 + lane] = acc[i][j0 + jj < CB ? j0 + jj : 0];
    __syncthreads();
    for (int it = wave; it < MB * JR; it += 4) {  // wave-uniform
      const int i = it / JR, jj = it % JR;
      if (j0 + jj >= CB) continue;
      const int blk = cb0 + j0 + jj;
      f32x4 v = red[((0 * MB + i) * JR + jj) * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) v = v + red[((w * MB + i) * JR + jj) * 64 + lane];
      float* tw = stage + wave * 256;
      float* part = e.part + (int64_t)slice * sh.M * sh.N;
      if (kind == EPI_F32) {
        store_tile<T, EPI_F32>(sh, e, mb0 + i, blk, v, nullptr, tw, nullptr, f32x4{}, f32x4{}, lane);
      } else if (kind == EPI_PARTIAL) {
        store_tile<T, EPI_PARTIAL>(sh, e, mb0 + i, blk, v, part, tw, nullptr, f32x4{}, f32x4{}, lane);
      } else if (kind == EPI_SWIGLU) {
        store_tile<T, EPI_SWIGLU>(sh, e, mb0 + i, blk, v, nullptr, tw, nullptr, f32x4{}, f32x4{}, lane);
      } else if (kind == EPI_QKV) {
        f32x4 cs = f32x4{1.f, 1.f, 1.f, 1.f}, sn = f32x4{0.f, 0.f, 0.f, 0.f};
        if (blk < 2 * e.H * (e.hd / 16)) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int lr = 16 * i + 4 * (lane >> 4) + r;
            if (16 * mb0 + lr < sh.M) {
              const int64_t ti = (int64_t)rm[lr].pos * (e.hd / 2) + 8 * (blk % (e.hd / 16)) + (lane & 7);
              cs[r] = e.rcos[ti];
              sn[r] = e.rsin[ti];
            }
          }
        }
        store_tile<T, EPI_QKV>(sh, e, mb0 + i, blk, v, nullptr, tw, rm + 16 * i, cs, sn, lane);
      }
    }
  }
}

// grid = (row blocks, runs, slices); workgroups [0, nbig) of a slice own CBA
// column blocks, the others CBA - 1.
template <typename T, int MB, int CBA, bool RM>
__global__ __launch_bounds__(256) void gemm_fp4_kernel(const GemmShape sh, const GemmEpi e, int64_t ldx,
                                                       const Fp4Shape w4, int kind, int nbig) {
  constexpr int JR = CBA < 32 / MB ? CBA : 32 / MB;
  __shared__ f32x4 red[4 * MB * JR * 64];
  __shared__ RowMeta rm[16 * MB];
  __shared__ __attribute__((aligned(16))) float stage[4 * 256];
  const int mb0 = blockIdx.x * MB, b = blockIdx.y, slice = blockIdx.z;
  if (kind == EPI_QKV && threadIdx.x < 16 * MB) {  // visible after the barrier that follows the k-loop
    const int row = 16 * mb0 + threadIdx.x;
    RowMeta t{-1, 0, -1};
    if (row < sh.M) t = RowMeta{e.kvoff[row], e.pos[row], e.qrow[row]};
    rm[threadIdx.x] = t;
  }
  if (b < nbig) {
    fp4_run<T, MB, CBA, RM>(sh, e, ldx, w4, kind, b * CBA, mb0, slice, red, rm, stage);
  } else {
    if constexpr (CBA > 1)
      fp4_run<T, MB, CBA - 1, RM>(sh, e, ldx, w4, kind, nbig * CBA + (b - nbig) * (CBA - 1), mb0, slice, red, rm,
                                  stage);
  }
}

constexpr int FP4_CB_MAX = 8;
constexpr int FP4_WGS = 256;

template <typename T, int MB, int CBA, bool RM>
void fp4_launch(const GemmShape& s, const GemmEpi& e, int64_t ldx, const Fp4Shape& w4, int kind, int runs, int nbig,
                hipStream_t st, hipEvent_t ea, hipEvent_t eb) {
  const dim3 grid((s.M + 16 * MB - 1) / (16 * MB), runs, s.splits);
  if (ea || eb)
    hipExtLaunchKernelGGL((gemm_fp4_kernel<T, MB, CBA, RM>), grid, dim3(256), 0, st, ea, eb, 0, s, e, ldx, w4, kind,
                          nbig);
  else
    hipLaunchKernelGGL((gemm_fp4_kernel<T, MB, CBA, RM>), grid, dim3(256), 0, st, s, e, ldx, w4, kind, nbig);
}

template <typename T, int MB, bool RM>
void fp4_mb(const GemmShape& s, const GemmEpi& e, int64_t ldx, const Fp4Shape& w4, int kind, hipStream_t st,
            hipEvent_t ea, hipEvent_t eb) {
  const int nbc = s.N / 16;
  const int runs = std::min(std::max((FP4_WGS + s.splits - 1) / s.splits, (nbc + FP4_CB_MAX - 1) / FP4_CB_MAX), nbc);
  const int run = (nbc + runs - 1) / runs, nbig = nbc - runs * (run - 1);
  switch (run) {
    case 1: fp4_launch<T, MB, 1, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 2: fp4_launch<T, MB, 2, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 3: fp4_launch<T, MB, 3, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 4: fp4_launch<T, MB, 4, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 5: fp4_launch<T, MB, 5, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 6: fp4_launch<T, MB, 6, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    case 7: fp4_launch<T, MB, 7, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
    default: fp4_launch<T, MB, 8, RM>(s, e, ldx, w4, kind, runs, nbig, st, ea, eb); break;
  }
}

template <typename T>
void fp4_t(const GemmShape& s, const GemmEpi& e, int64_t ldx, const Fp4Shape& w4, int kind, hipStream_t st,
           hipEvent_t ea, hipEvent_t eb) {
  if (s.M <= 16 && ldx > 0)
    fp4_mb<T, 1, true>(s, e, ldx, w4, kind, st, ea, eb);
  else if (s.M <= 16)
    fp4_mb<T, 1, false>(s, e, 0, w4, kind, st, ea, eb);
  else if (s.M <= 32)
    fp4_mb<T, 2, false>(s, e, 0, w4, kind, st, ea, eb);
  else
    fp4_mb<T, 4, false>(s, e, 0, w4, kind, st, ea, eb);
}

// Row-major x with a row stride into tiles, 16 bytes a thread; rows that do not
// start at 16 bytes are read element by element.
template <typename T>
__global__ __launch_bounds__(256) void tile_strided_kernel(const T* __restrict__ x, int64_t ldx, int M, int K,
                                                           T* __restrict__ dst, int mtiles, int aligned) {
  constexpr int VEC = ET<T>::VEC;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)M * (K / VEC)) return;
  const int r = (int)(i % M), q = (int)(i / M);
  const T* src = x + (int64_t)r * ldx + q * VEC;
  int4 v;
  if (aligned) {
    v = ld16(src);
  } else {
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int j = 0; j < VEC; ++j) e[j] = src[j];
  }
  st16(dst + tiled_index<T>(mtiles, r, q * VEC), v);
}

unsigned unit_blocks(const Fp4Shape& w4) { return (unsigned)((w4.codes_bytes / 1024 + 3) / 4); }

}  // namespace

int fp4_splits(int N, int K) { return gemm_pick_splits(N, K, DT_BF16); }

int64_t fp4_bytes(int N, int K) {
  const Fp4Shape s = fp4_shape(N, K, fp4_splits(N, K));
  return s.codes_bytes + s.codes_bytes / 16;
}

void launch_fp4_pack(int dtype, int kind, const void* s0, const void* s1, const void* s2, int64_t ldw, int N, int K,
                     void* dst, int H, int hd, hipStream_t st) {
  const Fp4Shape w4 = fp4_shape(N, K, fp4_splits(N, K));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(fp4_pack_kernel<bf16_t>, dim3(unit_blocks(w4)), dim3(256), 0, st, (const bf16_t*)s0,
                       (const bf16_t*)s1, (const bf16_t*)s2, ldw, kind, H, hd, w4, (uint8_t*)dst);
  else
    hipLaunchKernelGGL(fp4_pack_kernel<float>, dim3(unit_blocks(w4)), dim3(256), 0, st, (const float*)s0,
                       (const float*)s1, (const float*)s2, ldw, kind, H, hd, w4, (uint8_t*)dst);
}

void launch_fp4_unpack_rows(int dtype, const void* packed, int N, int K, void* dst, int64_t ldw, hipStream_t st) {
  const Fp4Shape w4 = fp4_shape(N, K, fp4_splits(N, K));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL((fp4_unpack_kernel<bf16_t, true>), dim3(unit_blocks(w4)), dim3(256), 0, st,
                       (const uint8_t*)packed, w4, (bf16_t*)dst, ldw);
  else
    hipLaunchKernelGGL((fp4_unpack_kernel<float, true>), dim3(unit_blocks(w4)), dim3(256), 0, st,
                       (const uint8_t*)packed, w4, (float*)dst, ldw);
}

void launch_tile_strided(int dtype, const void* x, int64_t ldx, int M, int K, void* dst, int mtiles, hipStream_t st) {
  const int es = dtype == DT_BF16 ? 2 : 4, VEC = 16 / es;
  const int aligned = ((uintptr_t)x & 15) == 0 && (M == 1 || ldx * es % 16 == 0);
  const dim3 grid((unsigned)(((int64_t)M * (K / VEC) + 255) / 256));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(tile_strided_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)x, ldx, M, K, (bf16_t*)dst,
                       mtiles, aligned);
  else
    hipLaunchKernelGGL(tile_strided_kernel<float>, grid, dim3(256), 0, st, (const float*)x, ldx, M, K, (float*)dst,
                       mtiles, aligned);
}

void launch_gemm_fp4(int dtype, const GemmShape& s, const GemmEpi& e, int64_t ldx, void* unpacked, hipStream_t st,
                     hipEvent_t ev_start, hipEvent_t ev_stop) {
  const Fp4Shape w4 = fp4_shape(s.N, s.K, s.splits);
  if (unpacked != nullptr) {
    hipLaunchKernelGGL((fp4_unpack_kernel<bf16_t, false>), dim3(unit_blocks(w4)), dim3(256), 0, st,
                       (const uint8_t*)s.W, w4, (bf16_t*)unpacked, (int64_t)0);
    GemmShape u = s;
    u.W = unpacked;
    (void)launch_gemm(dtype, u, e, st, ev_start, ev_stop);
    return;
  }
  const bool finish = s.splits > 1 && e.kind != EPI_PARTIAL;
  const int kind = finish ? EPI_PARTIAL : e.kind;
  if (dtype == DT_BF16)
    fp4_t<bf16_t>(s, e, ldx, w4, kind, st, ev_start, finish ? nullptr : ev_stop);
  else
    fp4_t<float>(s, e, ldx, w4, kind, st, ev_start, finish ? nullptr : ev_stop);
  if (finish) launch_gemm_finish(dtype, s, e, st, ev_stop);
}

bool gemm_fp4_unpacks(int dtype, int M, int N) { return dtype == DT_BF16 && N % 64 == 0 && M > FP4_DIRECT_ROWS; }
