// The C ABI's 4-bit operators (include/chimera.h): checks, workspaces and
// launches.  None allocates device memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "abi.h"
#include "chimera.h"
#include "kernels.h"
#include "ops.h"

namespace {

constexpr int FP4_MAX_ROWS = 4096;  // rows of a product: two prefill chunks

void check_matrix(int32_t N, int32_t K) {
  REQUIRE(N > 0 && N % 16 == 0 && K > 0 && K % 32 == 0, CHIMERA_EINVAL, "N must be a multiple of 16, K of 32");
  REQUIRE(N <= 1 << 20 && K <= 1 << 20, CHIMERA_EINVAL, "N and K are at most 2^20");
}

// Workspace of a product: tiled x, then the unpacked matrix where the launch
// takes the bf16 kernels, then the slices' partials.
struct GemmWs {
  int64_t x = 0, w = 0, part = 0;
  bool rows;  // x is read where it lies
  int64_t bytes() const { return x + w + part; }
};
GemmWs gemm_ws(int32_t dtype, int32_t M, int32_t N, int32_t K, bool readable) {
  GemmWs s;
  const int64_t es = (int64_t)esize(dtype);
  const bool unpack = gemm_fp4_unpacks(dtype, M, N, K);
  // A launch saved against reads of 64 bytes a row: at 64 rows 4096 x 22016 29.8 us
  // and 28.1 with the tiling launch, 4096 x 12288 22.0 and 20.0, 4096 x 4096 10.8
  // and 11.1.
  s.rows = M <= 32 && readable;
  if (!s.rows) s.x = round256((int64_t)mcap(M) * K * es);
  if (unpack) s.w = round256((int64_t)K * N * 2);
  const int parts = unpack ? gemm_partials(dtype, M, N, K, mcap(M) / 16, EPI_F32)
                           : (fp4_splits(N, K) > 1 ? fp4_splits(N, K) : 0);
  s.part = (int64_t)parts * M * N * 4;
  return s;
}

void check_cache(const chimera_kv4* c) {
  REQUIRE(c != nullptr && c->pool != nullptr && c->page_table != nullptr, CHIMERA_EINVAL, "null cache");
  REQUIRE(c->head_dim == 64 || c->head_dim == 128, CHIMERA_EINVAL, "head_dim must be 64 or 128");
  REQUIRE(c->n_heads >= 1 && c->n_heads <= 1024, CHIMERA_EINVAL, "n_heads in [1, 1024]");
  REQUIRE(c->page_size >= 1 && c->page_size <= 256, CHIMERA_EINVAL, "page_size in [1, 256]");
  REQUIRE(c->n_pages >= 1 && c->batch >= 1 && c->batch <= 65535 && c->max_pages >= 1, CHIMERA_EINVAL,
          "n_pages, batch and max_pages must be positive, batch at most 65535");
  REQUIRE((int64_t)c->max_pages * c->page_size <= (int64_t)1 << 30, CHIMERA_EINVAL, "more than 2^30 positions");
  check_aligned(c->pool, "pool");
  int64_t need = 0;
  if (chimera_kv4_bytes(c->n_pages, c->page_size, c->n_heads, c->head_dim, &need) != CHIMERA_OK)
    throw Err(CHIMERA_EINVAL, g_err);
  // groups of 32 values are named by 32 bits
  REQUIRE(need / 17 < (int64_t)1 << 32, CHIMERA_EINVAL, "pool over 68 GiB");
  REQUIRE(c->pool_bytes >= need, CHIMERA_ENOMEM, "pool too small");
}
Kv4View view(const chimera_kv4* c) {
  Kv4View v;
  v.page_stride = (int64_t)2 * c->n_heads * c->page_size * c->head_dim;
  v.codes = (uint8_t*)c->pool;
  v.scales = v.codes + (int64_t)c->n_pages * v.page_stride / 2;
  v.page_table = c->page_table;
  v.B = c->batch;
  v.max_pages = c->max_pages;
  v.n_pages = c->n_pages;
  v.ps = c->page_size;
  v.H = c->n_heads;
  v.hd = c->head_dim;
  return v;
}
void check_rows(const chimera_kv4* c, int32_t dtype, const void* k, const void* v, int64_t ld, const int32_t* seq,
                const int32_t* pos, int32_t rows) {
  check_cache(c);
  check_dtype(dtype);
  REQUIRE(rows >= 0, CHIMERA_EINVAL, "rows");
  REQUIRE(rows == 0 || (k && v && seq && pos), CHIMERA_EINVAL, "null argument");
  REQUIRE(ld >= (int64_t)c->n_heads * c->head_dim, CHIMERA_EINVAL, "row stride below n_heads * head_dim");
  REQUIRE((int64_t)rows * c->n_heads * c->head_dim / 4 < (int64_t)1 << 38, CHIMERA_EINVAL, "too many rows");
}

void check_queries(const chimera_kv4* c, int32_t n_heads, int32_t n_nodes) {
  check_cache(c);
  REQUIRE(n_heads >= 1 && n_heads <= 1024 && n_heads % c->n_heads == 0, CHIMERA_EINVAL,
          "n_heads must be a multiple of the cache's heads, at most 1024");
  REQUIRE(n_nodes >= 1 && n_nodes <= 64, CHIMERA_EINVAL, "n_nodes in [1, 64]");
}
int64_t attn_bytes(const chimera_kv4* c, int batch, int32_t n_heads, int32_t n_nodes) {
  return kv4_attn_bytes(batch, (int64_t)c->max_pages * c->page_size, n_heads, c->n_heads, c->head_dim, n_nodes);
}

}  // namespace

extern "C" {

chimera_status chimera_fp4_bytes(int32_t N, int32_t K, int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_matrix(N, K);
    *bytes = fp4_bytes(N, K);
  });
}

chimera_status chimera_fp4_pack(int32_t dtype, const void* w, int64_t ldw, int32_t N, int32_t K, void* packed,
                                int64_t packed_bytes, void* stream) {
  return guard([&] {
    check_dtype(dtype);
    REQUIRE(w && packed, CHIMERA_EINVAL, "null argument");
    check_matrix(N, K);
    REQUIRE(ldw >= N, CHIMERA_EINVAL, "ldw below N");
    check_aligned(packed, "packed");
    REQUIRE(packed_bytes >= fp4_bytes(N, K), CHIMERA_ENOMEM, "packed buffer too small");
    hipStream_t st = check_stream(stream);
    launch_fp4_pack(dtype, PACK_NATURAL, w, nullptr, nullptr, ldw, N, K, packed, 1, 64, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_fp4_unpack(int32_t dtype, const void* packed, int32_t N, int32_t K, void* w, int64_t ldw,
                                  void* stream) {
  return guard([&] {
    check_dtype(dtype);
    REQUIRE(w && packed, CHIMERA_EINVAL, "null argument");
    check_matrix(N, K);
    REQUIRE(ldw >= N, CHIMERA_EINVAL, "ldw below N");
    check_aligned(packed, "packed");
    hipStream_t st = check_stream(stream);
    launch_fp4_unpack_rows(dtype, packed, N, K, w, ldw, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_gemm_fp4_bytes(int32_t dtype, int32_t M, int32_t N, int32_t K, int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_dtype(dtype);
    REQUIRE(M >= 1 && M <= FP4_MAX_ROWS, CHIMERA_EINVAL, "M in [1, 4096]");
    check_matrix(N, K);
    // Fewer rows may leave more partials, where the more run on a kernel that sums
    // them: the route changes with whole 64-row blocks, and grows within one.
    *bytes = gemm_ws(dtype, M, N, K, false).bytes();
    for (int m = (M - 1) / 64 * 64; m > 0; m -= 64) *bytes = std::max(*bytes, gemm_ws(dtype, m, N, K, false).bytes());
  });
}

chimera_status chimera_gemm_fp4(int32_t dtype, const void* x, int64_t ldx, const void* packed, int32_t M, int32_t N,
                                int32_t K, float* y, int64_t ldy, void* ws, int64_t ws_bytes, void* stream) {
  return guard([&] {
    check_dtype(dtype);
    REQUIRE(x && packed && y, CHIMERA_EINVAL, "null argument");
    REQUIRE(M >= 1 && M <= FP4_MAX_ROWS, CHIMERA_EINVAL, "M in [1, 4096]");
    check_matrix(N, K);
    REQUIRE(ldx >= K && ldy >= N && ldy <= INT32_MAX, CHIMERA_EINVAL, "ldx below K, ldy below N, or ldy over 2^31 - 1");
    check_aligned(packed, "packed");
    const int64_t es = (int64_t)esize(dtype);
    const bool readable = ((uintptr_t)x & 15) == 0 && (M == 1 || ldx * es % 16 == 0);
    const GemmWs s = gemm_ws(dtype, M, N, K, readable);
    REQUIRE(s.bytes() == 0 || ws != nullptr, CHIMERA_EINVAL, "null workspace");
    REQUIRE(ws_bytes >= s.bytes(), CHIMERA_ENOMEM, "workspace too small");
    check_aligned(ws, "workspace");
    hipStream_t st = check_stream(stream);
    char* base = (char*)ws;
    GemmShape g;
    g.x_mtiles = mcap(M) / 16;
    g.M = M;
    g.W = packed;
    g.N = N;
    g.K = K;
    g.splits = fp4_splits(N, K);
    g.X = x;
    if (!s.rows) {
      launch_tile_strided(dtype, x, ldx, M, K, base, g.x_mtiles, st);
      g.X = base;
    }
    GemmEpi e;
    e.kind = EPI_F32;
    e.out_f = y;
    e.ldo = (int)ldy;
    e.part = (float*)(base + s.x + s.w);
    launch_gemm_fp4(dtype, g, e, s.rows ? ldx : 0, s.w ? base + s.x : nullptr, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_kv4_bytes(int32_t n_pages, int32_t page_size, int32_t n_heads, int32_t head_dim,
                                 int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    REQUIRE(n_pages >= 1, CHIMERA_EINVAL, "n_pages");
    REQUIRE(page_size >= 1 && page_size <= 256, CHIMERA_EINVAL, "page_size in [1, 256]");
    REQUIRE(n_heads >= 1 && n_heads <= 1024, CHIMERA_EINVAL, "n_heads in [1, 1024]");
    REQUIRE(head_dim == 64 || head_dim == 128, CHIMERA_EINVAL, "head_dim must be 64 or 128");
    const int64_t rows = (int64_t)n_pages * 2 * n_heads * page_size;
    *bytes = rows * (head_dim / 2 + head_dim / 32);
  });
}

chimera_status chimera_kv4_append(const chimera_kv4* cache, int32_t dtype, const void* k, const void* v, int64_t ld,
                                  const int32_t* seq, const int32_t* pos, int32_t rows, void* stream) {
  return guard([&] {
    check_rows(cache, dtype, k, v, ld, seq, pos, rows);
    hipStream_t st = check_stream(stream);
    if (rows == 0) return;
    launch_kv4_append(dtype, view(cache), k, v, ld, seq, pos, nullptr, rows, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_kv4_read(const chimera_kv4* cache, int32_t dtype, const int32_t* seq, const int32_t* pos,
                                int32_t rows, void* k_out, void* v_out, int64_t ld, void* stream) {
  return guard([&] {
    check_rows(cache, dtype, k_out, v_out, ld, seq, pos, rows);
    hipStream_t st = check_stream(stream);
    if (rows == 0) return;
    launch_kv4_read(dtype, view(cache), k_out, v_out, ld, seq, pos, rows, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_kv4_attn_bytes(const chimera_kv4* cache, int32_t n_heads, int32_t n_nodes, int64_t* bytes) {
  return guard([&] {
    check_queries(cache, n_heads, n_nodes);
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    // Fewer queries may leave groups where more leave supers: kv4_attn_units falls
    // with ceil(KV4_SUPER_WGS / blocks), and the size grows where that stays.
    *bytes = 0;
    for (int n = 1; n <= n_nodes; ++n) {
      const int per = kv4_attn_blocks(1, n_heads, cache->n_heads, n);
      if (n < n_nodes && kv4_attn_blocks(1, n_heads, cache->n_heads, n + 1) == per) continue;
      for (int b = cache->batch; b > 0;) {
        *bytes = std::max(*bytes, attn_bytes(cache, b, n_heads, n));
        const int factor = (KV4_SUPER_WGS + b * per - 1) / (b * per);
        b = std::min(b - 1, (KV4_SUPER_WGS - 1) / (per * factor));  // the most sequences with a larger one
      }
    }
  });
}

chimera_status chimera_kv4_attn(const chimera_kv4* cache, int32_t dtype, const void* q, int64_t ldq, const int32_t* n_b,
                                int32_t n_heads, const int32_t* parent, int32_t n_nodes, float scale, void* out,
                                int64_t ldo, void* ws, int64_t ws_bytes, void* stream) {
  return guard([&] {
    check_dtype(dtype);
    check_queries(cache, n_heads, n_nodes);
    REQUIRE(q && n_b && out && ws, CHIMERA_EINVAL, "null argument");
    REQUIRE(ws_bytes >= attn_bytes(cache, cache->batch, n_heads, n_nodes), CHIMERA_ENOMEM, "workspace too small");
    const int64_t es = (int64_t)esize(dtype), width = (int64_t)n_heads * cache->head_dim;
    REQUIRE(ldq >= width && ldo >= width, CHIMERA_EINVAL, "row stride below n_heads * head_dim");
    REQUIRE(ldq * es % 16 == 0, CHIMERA_EINVAL, "rows of q must start at multiples of 16 bytes");
    check_aligned(q, "q");
    check_aligned(ws, "workspace");
    REQUIRE(std::isfinite(scale) && std::fabs(scale) <= 0x1p127f, CHIMERA_EINVAL,
            "scale must be finite, at most 2^127 in magnitude");  // times log2(e) it still is
    Kv4AttnArgs a{};
    for (int u = 0; u < n_nodes; ++u) {
      const int p = parent ? parent[u] : u - 1;
      REQUIRE(u == 0 ? p == -1 : (p >= 0 && p < u), CHIMERA_EINVAL,
              "node 0 must be the root and a parent must precede its child");
      REQUIRE(u == 0 || a.tree.depth_of(p) < KV4_MAX_DEPTH, CHIMERA_EINVAL, "tree deeper than 15 levels below its root");
      a.tree.set(u, p);
      a.deepest = std::max(a.deepest, a.tree.depth_of(u));
    }
    hipStream_t st = check_stream(stream);
    a.c = view(cache);
    a.q = q;
    a.ldq = ldq;
    a.out = out;
    a.ldo = ldo;
    a.n_b = n_b;
    a.Hq = n_heads;
    a.N = n_nodes;
    a.scale = scale;
    const int64_t cap = (int64_t)cache->max_pages * cache->page_size;
    a.blocks = kv4_attn_blocks(cache->batch, n_heads, cache->n_heads, n_nodes);
    a.units = kv4_attn_units(cap, a.blocks);
    a.one = kv4_attn_one(cap);
    a.part_o = (float*)ws;
    a.part_ml = a.part_o + (int64_t)cache->batch * a.units * n_nodes * n_heads * cache->head_dim;
    launch_kv4_attn(dtype, a, st);
    HIPCK(hipGetLastError());
  });
}

}  // extern "C"
