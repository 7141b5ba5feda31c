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
// A class's last quad is whole too, and its padding (zeros) is stored and streamed:
// nothing where a slice is a multiple of 512 values, 12% at 11008 x 4096 (four slices
// of 86 k-blocks), 20% at 5120 x 5120, 4% at 13824 x 5120, 100% at K = 256.
#include <hip/hip_ext.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "fp4.h"
#include "gemm_epilogue.h"
#include "kernels.h"

namespace {

constexpr int DIES = 8;  // each with an L2 of its own
constexpr int FP4_WGS = 256;  // a workgroup a CU

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

// One wave a unit; a group's 32 values lie in the four lanes of a column.  A lane
// reads an element of each of its rows, 16 columns of a row side by side: 4096 x
// 22016 of bf16 62 us, 3.7 TB/s; weights are packed once.
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

// The values: row-major [K][N] (ROWS; 4096 x 22016 96 us, stores of 16 columns a
// row), or bf16 in the layout of the bf16 kernels (kernels_gemm.hip; N a multiple of
// 64).
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

// X rows of a launch: tiled (fragment order, x_mtiles 16-row tiles), or where they
// lie (RM, row stride ldx).
template <typename T, bool RM, int MB>
struct XRows {
  const T* base;
  int64_t step;         // elements from one 32-wide k-block to the next
  int64_t row[RM ? MB : 1];  // RM: from the first tile's row of this lane to those of the others
  __device__ __forceinline__ XRows(const GemmShape& sh, int64_t ldx, int mb0, int lane) {
    const int g = lane >> 4, r = lane & 15;
    if constexpr (RM) {  // rows past M repeat the last one; they are not stored
      base = (const T*)sh.X + 8 * g;
      step = 32;
#pragma unroll
      for (int i = 0; i < MB; ++i) row[i] = (int64_t)min(16 * (mb0 + i) + r, sh.M - 1) * ldx;
    } else {
      step = (int64_t)sh.x_mtiles * 64 * 8;
      if constexpr (sizeof(T) == 2)
        base = (const T*)sh.X + ((int64_t)mb0 * 64 + lane) * 8;
      else  // two k-blocks of 16: lanes of pieces 2 (g & 1) and 2 (g & 1) + 1 of block g >> 1
        base = (const T*)sh.X + (((int64_t)(g >> 1) * sh.x_mtiles + mb0) * 64 + 32 * (g & 1) + r) * 4;
    }
  }
  __device__ __forceinline__ void load(int kb, int i, Frag32<T>& f) const {
    const T* p = base + (int64_t)kb * step + (RM ? row[RM ? i : 0] : i * 64 * (int64_t)(16 / sizeof(T)));
    f.v[0] = ld16(p);
    if constexpr (sizeof(T) == 4) f.v[1] = ld16(p + (RM ? 4 : 16 * 4));
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

// A 16x16 output tile: rows of tile mb, column block blk; rm: its rows' targets.
template <typename T>
__device__ __forceinline__ void store_output(const GemmShape& sh, const GemmEpi& e, int kind, int mb, int blk,
                                             int slice, f32x4 v, float* tw, const RowMeta* rm, int lane) {
  if (kind == EPI_F32) {
    store_tile<T, EPI_F32>(sh, e, mb, blk, v, nullptr, tw, nullptr, f32x4{}, f32x4{}, lane);
  } else if (kind == EPI_PARTIAL) {
    float* part = e.part + (int64_t)slice * sh.M * sh.N;
    store_tile<T, EPI_PARTIAL>(sh, e, mb, blk, v, part, tw, nullptr, f32x4{}, f32x4{}, lane);
  } else if (kind == EPI_SWIGLU) {
    store_tile<T, EPI_SWIGLU>(sh, e, mb, blk, v, nullptr, tw, nullptr, f32x4{}, f32x4{}, lane);
  } else if (kind == EPI_QKV) {
    f32x4 cs = f32x4{1.f, 1.f, 1.f, 1.f}, sn = f32x4{0.f, 0.f, 0.f, 0.f};
    if (blk < 2 * e.H * (e.hd / 16)) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int lr = 4 * (lane >> 4) + r;
        if (16 * mb + lr < sh.M) {
          const int64_t ti = (int64_t)rm[lr].pos * (e.hd / 2) + 8 * (blk % (e.hd / 16)) + (lane & 7);
          cs[r] = e.rcos[ti];
          sn[r] = e.rsin[ti];
        }
      }
    }
    store_tile<T, EPI_QKV>(sh, e, mb, blk, v, nullptr, tw, rm, cs, sn, lane);
  }
}
// The QKV epilogue's targets of `rows` rows from `first`, into LDS.
__device__ __forceinline__ void row_targets(const GemmShape& sh, const GemmEpi& e, int first, int rows, RowMeta* rm) {
  if ((int)threadIdx.x >= rows) return;
  const int row = first + threadIdx.x;
  RowMeta t{-1, 0, -1};
  if (row < sh.M) t = RowMeta{e.kvoff[row], e.pos[row], e.qrow[row]};
  rm[threadIdx.x] = t;
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
  const XRows<T, RM, MB> X(sh, ldx, mb0, lane);
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
      store_output<T>(sh, e, kind, mb0 + i, blk, slice, v, stage + wave * 256, rm + 16 * i, lane);
    }
  }
}

// grid = (row blocks, runs, slices); workgroups [0, nbig) of a slice own CBA
// column blocks, the others CBA - 1.  mapped: the row blocks of a run go to one
// die (dealt round-robin by linear id), whose L2 then has their weights (256 rows,
// 4096 x 12288: 43.0 -> 37.4 us).
//
// A quad of weights (1 KiB of codes a wave) is requested while the quad before it is
// converted, straight from memory: nothing of W is read twice by a workgroup.  Up
// to 16 rows it is bound by that stream (1 row of 4096 x 22016 11.7 us, 4.1 TB/s);
// from 64 rows on by each CU's intake of its activations (64 rows of 4096 x 22016
// 23.5 us, of 4096 x 12288 with their tiling 18.4; 2.5 TB/s of memory, the MFMA busy
// 16% and the VALU 12% of the time), which longer runs of columns would take in less
// often but do not fit the registers with.
template <typename T, int MB, int CBA, bool RM>
__global__ __launch_bounds__(256) void gemm_fp4_kernel(const GemmShape sh, const GemmEpi e, int64_t ldx,
                                                       const Fp4Shape w4, int kind, int nbig, int mapped) {
  constexpr int JR = CBA < 32 / MB ? CBA : 32 / MB;
  __shared__ f32x4 red[4 * MB * JR * 64];
  __shared__ RowMeta rm[16 * MB];
  __shared__ __attribute__((aligned(16))) float stage[4 * 256];
  int rb = blockIdx.x, b = blockIdx.y, slice = blockIdx.z;
  if (MB > 1 && mapped) {  // uniform
    const int X = gridDim.x, Y = gridDim.y, id = blockIdx.x + X * (blockIdx.y + Y * blockIdx.z);
    const int k = id / DIES, r = k / X * DIES + id % DIES;
    rb = k % X;
    b = r % Y;
    slice = r / Y;
  }
  const int mb0 = rb * MB;
  if (kind == EPI_QKV) row_targets(sh, e, 16 * mb0, 16 * MB, rm);  // visible after the barrier behind the k-loop
  if (b < nbig) {
    fp4_run<T, MB, CBA, RM>(sh, e, ldx, w4, kind, b * CBA, mb0, slice, red, rm, stage);
  } else {
    if constexpr (CBA > 1)
      fp4_run<T, MB, CBA - 1, RM>(sh, e, ldx, w4, kind, nbig * CBA + (b - nbig) * (CBA - 1), mb0, slice, red, rm,
                                  stage);
  }
}

constexpr int FP4_ROWS_BYTES = 112 << 10;     // rows of the kernel below, next to its sums in LDS
constexpr int FP4_TWO_ROWS_BYTES = 47 << 10;  // with two workgroups on a CU

// Split products of up to 16 rows whose sum nobody else finishes: a workgroup
// owns one column block and the whole reduction, S slices of four waves (one a
// class) side by side, and the slices meet in LDS, not in a finishing launch.
// Its share is short (35 KB of 4096 x 16), a quarter of the bf16 kernels'.  The
// rows are staged in LDS, only the ones there are; a thread's first pieces are
// requested before its weights, since loads return in order and the weights
// need not be waited for there.  One row of 4096 x 4096 5.4 us with its launch in a
// graph (floor 1.7): a start, a round trip for rows and weights and two barriers.
template <typename T, int S, bool RM>
__global__ __launch_bounds__(256 * S) void gemm_fp4_whole_kernel(const GemmShape sh, const GemmEpi e, int64_t ldx,
                                                                 const Fp4Shape w4) {
  constexpr int PF = 4, XU = 2;           // quads in flight; pieces of x a thread requests first
  constexpr int J = sizeof(T) / 2;        // 16-byte pieces of eight values
  extern __shared__ int4 xs[];
  __shared__ f32x4 red[GEMM_MAX_SPLITS * 4 * 64];
  __shared__ __attribute__((aligned(16))) float stage[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), cls = wave & 3;
  const int g = lane >> 4, r = min(lane & 15, sh.M - 1);  // rows past M repeat the last one; they are not stored
  const int nk = cls < w4.kps ? (w4.kps - cls + 3) / 4 : 0, nq = (nk + 3) / 4;
  // piece (kb, g, half) of row q goes to ((4 kb + g) J + half) M + q
  const int total = sh.K / ET<T>::VEC * sh.M;
  auto piece = [&](int i) {
    const int q = i % sh.M, k = i / sh.M * ET<T>::VEC;
    return RM ? ld16((const T*)sh.X + (int64_t)q * ldx + k) : ld16((const T*)sh.X + tiled_index<T>(sh.x_mtiles, q, k));
  };
  int4 xr[XU];
#pragma unroll
  for (int t = 0; t < XU; ++t)
    if (tid + t * 256 * S < total) xr[t] = piece(tid + t * 256 * S);
  int4 bc[PF];
  uint32_t bs[PF];
  const uint8_t* codes = nullptr;
  const uint8_t* scales = nullptr;
  auto load_w = [&](int slot, int q) {
    bc[slot] = ld16_nt(codes + (int64_t)q * 1024);
    bs[slot] = *reinterpret_cast<const uint32_t*>(scales + (int64_t)q * 64);
  };
  auto start = [&](int slice) {
    const int64_t u = fp4_unit(w4, blockIdx.x, slice, cls);
    codes = (const uint8_t*)sh.W + u * 1024 + lane * 16;
    scales = (const uint8_t*)sh.W + w4.codes_bytes + u * 64 + (lane & 15) * 4;
#pragma unroll
    for (int t = 0; t < PF; ++t)
      if (t < nq) load_w(t, t);
  };
  start(wave / 4);
#pragma unroll
  for (int t = 0; t < XU; ++t)
    if (tid + t * 256 * S < total) xs[tid + t * 256 * S] = xr[t];
  for (int i = tid + XU * 256 * S; i < total; i += 256 * S) xs[i] = piece(i);
  __syncthreads();
  for (int sl = wave / 4; sl < w4.splits; sl += S) {
    if (sl >= S) start(sl);
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
    const int4* x = xs + ((int64_t)(sl * w4.kps + cls) * 4 + g) * J * sh.M + r;
    const int step = 16 * J * sh.M;  // four k-blocks on
    for (int q0 = 0; q0 < nq; q0 += PF) {
#pragma unroll
      for (int t = 0; t < PF; ++t) {
        if (q0 + t >= nq) break;  // wave-uniform
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = 4 * (q0 + t) + i;
          if (k >= nk) break;
          Frag32<T> xf, w;
#pragma unroll
          for (int h = 0; h < J; ++h) xf.v[h] = x[k * step + h * sh.M];
          w.from_fp4(word(bc[t], i), fp4_scale((bs[t] >> (8 * i)) & 255));
          acc = mfma32<T>(xf, w, acc);
        }
        if (q0 + t + PF < nq) load_w(t, q0 + t + PF);
      }
    }
    red[(sl * 4 + cls) * 64 + lane] = acc;
  }
  __syncthreads();
  if (wave != 0) return;
  f32x4 v;
  for (int sl = 0; sl < w4.splits; ++sl) {  // classes in class order, slices in slice order
    f32x4 t = red[(sl * 4) * 64 + lane];
#pragma unroll
    for (int c = 1; c < 4; ++c) t = t + red[(sl * 4 + c) * 64 + lane];
    v = sl == 0 ? t : v + t;
  }
  store_tile<T, EPI_F32>(sh, e, 0, blockIdx.x, v, nullptr, stage, nullptr, f32x4{}, f32x4{}, lane);
}

// FP4_WHOLE: the kernel above, where the rows fit LDS.  FP4_ROWS: blocks of rows
// read where they lie (at most 32).  FP4_BLOCKS: from tiles.
enum Fp4Route { FP4_BLOCKS, FP4_ROWS, FP4_WHOLE };
// Whether a workgroup a column block is the faster form of such a product, against
// the slices in workgroups of their own and a finishing launch.  The first takes as
// long as K weights and M K activations take through one CU, whatever N; the second
// 1.2 us longer to start, and then K N through all CUs.  So up to a column block a CU
// the first wins where K (A + B M - N) stays below C; past that, with a second
// block's rows beside the first's in LDS, where K (A + M) stays below C N.  The
// constants fit 1534 measured sizes (N 16 to 8176, K 1024 to 57344, 1 to 16 rows,
// weights from memory, calls in a graph), where the form taken is 0.2% (bf16) and
// 0.6% (fp32) slower than the better one on average and 9% and 21% at most.  bf16,
// us, workgroup a block / slices: 1 row of 2048 x 256 3.5 / 3.9, 4096 x 256 5.0 / 4.5,
// 4096 x 4096 5.4 / 6.8, 8192 x 2048 6.7 / 6.6, 28672 x 4096 17.2 / 17.1, 57344 x 4096
// 30.7 / 26.5, 8192 x 5120 8.9 / 9.7, 13824 x 5120 14.2 / 12.3; 16 rows of 1024 x 2048
// 4.2 / 4.9, 2560 x 2048 6.6 / 6.2; 4 rows of 8192 x 5120 (one block's rows) 15.9 / 9.8.
bool fp4_whole_pays(int dtype, int64_t M, int64_t N, int64_t K) {
  const bool bf = dtype == DT_BF16;
  const int64_t bytes = M * K * (bf ? 2 : 4);
  if (N <= 16 * FP4_WGS) {
    if (bytes > FP4_ROWS_BYTES) return false;
    return bf ? K * (3000 + 200 * M - N) < 10000000 && K <= 8 * N + 2048 : K * (3400 + 250 * M - N) < 4000000;
  }
  return bytes <= FP4_TWO_ROWS_BYTES && (bf ? K * (2 + M) < 7 * N : K * (4 + M) < 2 * N);
}
Fp4Route fp4_route(int dtype, int M, int N, int K, int splits, int kind, int64_t ldx) {
  if (M <= 16 && splits > 1 && kind == EPI_F32 && fp4_whole_pays(dtype, M, N, K)) return FP4_WHOLE;
  return ldx > 0 ? FP4_ROWS : FP4_BLOCKS;
}

constexpr int FP4_CB_MAX = 8;

// Column runs of a slice: FP4_WGS workgroups' worth, at most FP4_CB_MAX blocks
// long; the first `big` runs have `run` blocks, the others one less.
struct Fp4Runs {
  int runs, run, big;
};
Fp4Runs fp4_runs(int nbc, int splits) {
  Fp4Runs r;
  r.runs = std::min(std::max((FP4_WGS + splits - 1) / splits, (nbc + FP4_CB_MAX - 1) / FP4_CB_MAX), nbc);
  r.run = (nbc + r.runs - 1) / r.runs;
  r.big = nbc - r.runs * (r.run - 1);
  return r;
}

struct Fp4Launch {
  const GemmShape& s;
  const GemmEpi& e;
  int64_t ldx;
  Fp4Shape w4;
  int kind;
  hipStream_t st;
  hipEvent_t ea, eb;

  template <typename... A, typename K>
  void go(K kernel, dim3 grid, int threads, size_t lds, A... args) const {
    if (ea || eb)
      hipExtLaunchKernelGGL(kernel, grid, dim3(threads), lds, st, ea, eb, 0, args...);
    else
      hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, st, args...);
  }
  // f(column blocks of a long run)
  template <class F>
  static void by_run(int run, F&& f) {
    switch (run) {
      case 1: f(std::integral_constant<int, 1>{}); break;
      case 2: f(std::integral_constant<int, 2>{}); break;
      case 3: f(std::integral_constant<int, 3>{}); break;
      case 4: f(std::integral_constant<int, 4>{}); break;
      case 5: f(std::integral_constant<int, 5>{}); break;
      case 6: f(std::integral_constant<int, 6>{}); break;
      case 7: f(std::integral_constant<int, 7>{}); break;
      default: f(std::integral_constant<int, 8>{}); break;
    }
  }
  template <typename T, int MB, bool RM>
  void blocks() const {
    const Fp4Runs r = fp4_runs(s.N / 16, s.splits);
    const dim3 grid((s.M + 16 * MB - 1) / (16 * MB), r.runs, s.splits);
    const int mapped = grid.x > 1 && r.runs * s.splits % DIES == 0;
    by_run(r.run, [&](auto cb) {
      go(gemm_fp4_kernel<T, MB, decltype(cb)::value, RM>, grid, 256, 0, s, e, ldx, w4, kind, r.big, mapped);
    });
  }
  template <typename T, bool RM>
  void whole() const {
    const dim3 grid(s.N / 16);
    const size_t lds = (size_t)s.M * s.K * sizeof(T);
    // sixteen waves a column block, eight where two workgroups a CU are wanted
    if (s.splits >= 4 && s.N / 16 <= FP4_WGS)
      go(gemm_fp4_whole_kernel<T, 4, RM>, grid, 1024, lds, s, e, ldx, w4);
    else
      go(gemm_fp4_whole_kernel<T, 2, RM>, grid, 512, lds, s, e, ldx, w4);
  }
  template <typename T>
  void run(Fp4Route route) const {
    if (route == FP4_WHOLE)
      ldx > 0 ? whole<T, true>() : whole<T, false>();
    else if (route == FP4_ROWS && s.M <= 16)
      blocks<T, 1, true>();
    else if (route == FP4_ROWS)
      blocks<T, 2, true>();
    else if (s.M <= 16)
      blocks<T, 1, false>();
    else if (s.M <= 32)
      blocks<T, 2, false>();
    else
      blocks<T, 4, false>();
  }
};

// Row-major x with a row stride into tiles: a wave a tile, a lane its 16 bytes (a
// row's four pieces of a k-block lie side by side); rows that do not start at 16
// bytes are read element by element.
template <typename T>
__global__ __launch_bounds__(256) void tile_strided_kernel(const T* __restrict__ x, int64_t ldx, int M, int kblocks,
                                                           int used, T* __restrict__ dst, int mtiles, int aligned) {
  constexpr int VEC = ET<T>::VEC;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= kblocks * used) return;
  const int kb = t / used, mb = t % used, r = 16 * mb + (lane & 15);
  if (r >= M) return;
  const T* src = x + (int64_t)r * ldx + kb * 4 * VEC + (lane >> 4) * VEC;
  int4 v;
  if (aligned) {
    v = ld16(src);
  } else {
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int j = 0; j < VEC; ++j) e[j] = src[j];
  }
  st16(dst + (((int64_t)kb * mtiles + mb) * 64 + lane) * VEC, v);
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
  const int kblocks = K / (4 * VEC), used = (M + 15) / 16;
  const dim3 grid((unsigned)((kblocks * used + 3) / 4));
  if (dtype == DT_BF16)
    hipLaunchKernelGGL(tile_strided_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)x, ldx, M, kblocks, used,
                       (bf16_t*)dst, mtiles, aligned);
  else
    hipLaunchKernelGGL(tile_strided_kernel<float>, grid, dim3(256), 0, st, (const float*)x, ldx, M, kblocks, used,
                       (float*)dst, mtiles, aligned);
}

void launch_gemm_fp4(int dtype, const GemmShape& s, const GemmEpi& e, int64_t ldx, void* unpacked, hipStream_t st,
                     hipEvent_t ev_start, hipEvent_t ev_stop) {
  const Fp4Shape w4 = fp4_shape(s.N, s.K, s.splits);
  if (unpacked != nullptr) {
    const Fp4Launch first{s, e, 0, w4, e.kind, st, ev_start, nullptr};  // the events span both launches
    first.go(fp4_unpack_kernel<bf16_t, false>, dim3(unit_blocks(w4)), 256, 0, (const uint8_t*)s.W, w4,
             (bf16_t*)unpacked, (int64_t)0);
    GemmShape u = s;
    u.W = unpacked;
    (void)launch_gemm(dtype, u, e, st, nullptr, ev_stop);
    return;
  }
  const Fp4Route route = fp4_route(dtype, s.M, s.N, s.K, s.splits, e.kind, ldx);
  const bool finish = s.splits > 1 && e.kind != EPI_PARTIAL && route != FP4_WHOLE;
  const Fp4Launch l{s, e, ldx, w4, finish ? (int)EPI_PARTIAL : e.kind, st, ev_start, finish ? nullptr : ev_stop};
  if (dtype == DT_BF16)
    l.run<bf16_t>(route);
  else
    l.run<float>(route);
  if (finish) launch_gemm_finish(dtype, s, e, st, ev_stop);
}

int gemm_fp4_direct_rows(int N, int K) {
  const int64_t weights = (int64_t)N * K;
  return weights >= 12 << 20 ? 384 : (weights >= 1 << 20 ? 768 : 2048);
}
bool gemm_fp4_unpacks(int dtype, int M, int N, int K) {
  return dtype == DT_BF16 && N % 64 == 0 && M > gemm_fp4_direct_rows(N, K);
}
