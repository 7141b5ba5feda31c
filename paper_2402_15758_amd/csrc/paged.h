// A plain paged KV cache (chimera_paged) as the kernels see it: rows of head_dim
// values in the order [page][K | V][head][slot].  A row is named by its index, 32
// bits for every pool the host accepts.
#pragma once
#include "kernels.h"

// Quotient by a number d in [1, 256] without a division.  With 2^k >= d and m =
// ceil(2^(30 + k) / d), m d = 2^(30 + k) + e, e < d, so floor(n m / 2^(30 + k)) is
// floor(n / d) while n e < 2^(30 + k): for every n < 2^30.  m <= 2^31.
struct PagedDiv {
  uint32_t m;
  int sh, d;
  explicit PagedDiv(int by) : sh(30), d(by) {
    while ((1 << (sh - 30)) < d) ++sh;
    m = (uint32_t)((((uint64_t)1 << sh) + d - 1) / d);
  }
  PagedDiv() : m(0), sh(0), d(0) {}
  __host__ __device__ __forceinline__ int quot(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> sh); }
};

struct PagedView {
  void* pool;
  const int* page_table;    // [B][max_pages]
  PagedDiv ps;
  int B, max_pages, n_pages, H, hd;
  int cap;                  // max_pages ps
  uint32_t page_rows;       // rows of a page: 2 H ps
};
constexpr uint32_t PAGED_NONE = 0xffffffffu;

// Row of position p of sequence b (head 0, K), PAGED_NONE where the cache has no
// such slot: a position outside the table, a page outside the pool.
__device__ __forceinline__ uint32_t paged_row(const PagedView& c, const int* __restrict__ ptab, int p) {
  if (p < 0 || p >= c.cap) return PAGED_NONE;
  const int pi = c.ps.quot(p);
  const int page = ptab[pi];
  if (page < 0 || page >= c.n_pages) return PAGED_NONE;
  return (uint32_t)page * c.page_rows + (uint32_t)(p - pi * c.ps.d);
}

// ---- rows with their rotation (kernels_paged.hip) --------------------------------
struct RopeArgs {
  int pairs;                // of a head: rot_dim / 2
  int scaling;              // 0 none, 1 linear, 2 ramp
  float base, factor, low, high, gain;
  int original;
};
// table [positions][pairs] of (cos, sin), float32
void launch_rope_table(const RopeArgs& r, void* table, int positions, hipStream_t st);

struct AppendArgs {
  const void *q, *k, *v;    // rows ld apart, heads of hd
  int64_t ld;
  void* q_out;              // rows ldo apart, of the cache's type
  int64_t ldo;
  const int *seq, *pos;
  const float2* table;      // [positions][pairs]
  const float *q_gain, *k_gain;  // [hd], nullptr: not normalised
  float eps;
  int Hq, rows;
  int pairs, cross, positions;   // 0 pairs: not rotated; cross: pairs (i, i + pairs), else neighbours
};
void launch_paged_append(int dtype, int held, const PagedView& c, const AppendArgs& a, hipStream_t st);

// ---- attention (kernels_paged_attn.hip) ------------------------------------------
struct PagedAttnArgs {
  const void* q;            // [rows][ldq], heads of hd
  int64_t ldq;
  void* out;
  int64_t ldo;
  const int* row0;          // [B + 1] first rows, nullptr: row b is sequence b's only one
  const int* n_b;           // [B] positions before them
  int rows, Hq, group;      // group = Hq / H
  int window, sinks;        // window 0: every position
  float scale2;             // |scale| log2(e)
  int flip;                 // scale < 0: queries are negated
  // a launch's own: parts of a block's positions at most and tiles of one at least, blocks
  // of queries of one cache head, those of each sequence (0: as its rows take)
  int splits, least, slots, per;
  float* part_o;            // [slots][H][splits][block][hd]
  float* part_ml;           // [slots][H][splits][block][2]
};
// Partials of a call, and of any with fewer rows or sequences.
int64_t paged_attn_bytes(int64_t cap, int rows, int batch, int group, int H, int hd, int es);
void launch_paged_attn(int dtype, const PagedView& c, PagedAttnArgs a, void* ws, hipStream_t st);
