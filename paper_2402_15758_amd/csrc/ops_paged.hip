// The C ABI's operators over a plain paged cache and the verification of drafted
// tokens (include/chimera.h): checks, workspaces and launches.  None allocates device
// memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "abi.h"
#include "accept.h"
#include "chimera.h"
#include "kernels.h"
#include "ops.h"
#include "paged.h"

namespace {

int64_t paged_bytes(const chimera_paged* c) {
  return (int64_t)c->n_pages * 2 * c->n_heads * c->page_size * c->head_dim * (int64_t)esize(c->dtype);
}
void check_shape(int32_t n_pages, int32_t page_size, int32_t n_heads, int32_t head_dim, int32_t dtype) {
  check_dtype(dtype);
  REQUIRE(n_pages >= 1, CHIMERA_EINVAL, "n_pages");
  REQUIRE(page_size >= 1 && page_size <= 256, CHIMERA_EINVAL, "page_size in [1, 256]");
  REQUIRE(n_heads >= 1 && n_heads <= 1024, CHIMERA_EINVAL, "n_heads in [1, 1024]");
  REQUIRE(head_dim == 64 || head_dim == 128, CHIMERA_EINVAL, "head_dim must be 64 or 128");
  // rows are named by 31 bits
  REQUIRE((int64_t)n_pages * 2 * n_heads * page_size < (int64_t)1 << 31, CHIMERA_EINVAL, "pool over 2^31 rows");
}
void check_paged(const chimera_paged* c) {
  REQUIRE(c != nullptr && c->pool != nullptr && c->page_table != nullptr, CHIMERA_EINVAL, "null cache");
  check_shape(c->n_pages, c->page_size, c->n_heads, c->head_dim, c->dtype);
  REQUIRE(c->batch >= 1 && c->batch <= 65535 && c->max_pages >= 1, CHIMERA_EINVAL,
          "batch and max_pages must be positive, batch at most 65535");
  REQUIRE((int64_t)c->max_pages * c->page_size <= (int64_t)1 << 30, CHIMERA_EINVAL, "more than 2^30 positions");
  check_aligned(c->pool, "pool");
  REQUIRE(c->pool_bytes >= paged_bytes(c), CHIMERA_ENOMEM, "pool too small");
}
PagedView view(const chimera_paged* c) {
  PagedView v;
  v.pool = c->pool;
  v.page_table = c->page_table;
  v.ps = PagedDiv(c->page_size);
  v.B = c->batch;
  v.max_pages = c->max_pages;
  v.n_pages = c->n_pages;
  v.H = c->n_heads;
  v.hd = c->head_dim;
  v.cap = c->max_pages * c->page_size;
  v.page_rows = (uint32_t)(2 * c->n_heads * c->page_size);
  return v;
}

void check_rope(const chimera_rope* r) {
  REQUIRE(r != nullptr, CHIMERA_EINVAL, "null rope");
  REQUIRE(r->rot_dim >= 2 && r->rot_dim <= 128 && r->rot_dim % 2 == 0, CHIMERA_EINVAL, "rot_dim: even, in [2, 128]");
  REQUIRE(r->layout == CHIMERA_ROPE_HALF || r->layout == CHIMERA_ROPE_PAIRS, CHIMERA_EINVAL, "rope layout");
  REQUIRE(r->max_positions >= 1 && r->max_positions <= 1 << 24, CHIMERA_EINVAL, "max_positions in [1, 2^24]");
  REQUIRE(std::isfinite(r->base) && r->base > 1.f, CHIMERA_EINVAL, "base must be finite, above 1");
  REQUIRE(std::isfinite(r->gain), CHIMERA_EINVAL, "gain must be finite");
  REQUIRE(r->scaling >= CHIMERA_ROPE_NONE && r->scaling <= CHIMERA_ROPE_RAMP, CHIMERA_EINVAL, "rope scaling");
  if (r->scaling != CHIMERA_ROPE_NONE)
    REQUIRE(std::isfinite(r->factor) && r->factor > 0.f, CHIMERA_EINVAL, "factor must be finite and positive");
  if (r->scaling == CHIMERA_ROPE_RAMP)
    REQUIRE(r->original_positions >= 1 && std::isfinite(r->low) && std::isfinite(r->high) && r->low >= 0.f &&
                r->high > r->low,
            CHIMERA_EINVAL, "a ramp needs original_positions and 0 <= low < high");
}
int64_t rope_bytes(const chimera_rope* r) { return (int64_t)r->max_positions * (r->rot_dim / 2) * 8; }

void check_heads(const chimera_paged* c, int32_t n_heads) {
  REQUIRE(n_heads >= 1 && n_heads <= 1024 && n_heads % c->n_heads == 0, CHIMERA_EINVAL,
          "n_heads must be a multiple of the cache's heads, at most 1024");
}
void check_attn_rows(const chimera_paged* c, int32_t n_heads, int32_t rows) {
  check_paged(c);
  check_heads(c, n_heads);
  // a launch's threads are counted in 32 bits
  REQUIRE(rows >= 0 && (int64_t)rows * n_heads <= (int64_t)1 << 26, CHIMERA_EINVAL, "rows * n_heads in [0, 2^26]");
  REQUIRE((int64_t)c->batch * n_heads <= (int64_t)1 << 23, CHIMERA_EINVAL, "batch * n_heads is at most 2^23");
}

void check_tree(int32_t batch, int32_t n_nodes, int32_t vocab) {
  REQUIRE(n_nodes >= 1 && n_nodes <= 64, CHIMERA_EINVAL, "n_nodes in [1, 64]");
  REQUIRE(batch >= 1 && batch <= 65535, CHIMERA_EINVAL, "batch in [1, 65535]");
  REQUIRE(vocab >= 1 && vocab <= 1 << 24, CHIMERA_EINVAL, "vocab in [1, 2^24]");
}

}  // namespace

extern "C" {

chimera_status chimera_paged_bytes(int32_t n_pages, int32_t page_size, int32_t n_heads, int32_t head_dim, int32_t dtype,
                                   int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_shape(n_pages, page_size, n_heads, head_dim, dtype);
    chimera_paged c{};
    c.n_pages = n_pages;
    c.page_size = page_size;
    c.n_heads = n_heads;
    c.head_dim = head_dim;
    c.dtype = dtype;
    *bytes = paged_bytes(&c);
  });
}

chimera_status chimera_rope_bytes(const chimera_rope* rope, int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_rope(rope);
    *bytes = rope_bytes(rope);
  });
}

chimera_status chimera_rope_table(const chimera_rope* rope, void* table, int64_t table_bytes, void* stream) {
  return guard([&] {
    check_rope(rope);
    REQUIRE(table != nullptr, CHIMERA_EINVAL, "null table");
    check_aligned(table, "table");
    REQUIRE(table_bytes >= rope_bytes(rope), CHIMERA_ENOMEM, "table too small");
    hipStream_t st = check_stream(stream);
    RopeArgs r{};
    r.pairs = rope->rot_dim / 2;
    r.scaling = rope->scaling;
    r.base = rope->base;
    r.factor = rope->factor;
    r.low = rope->low;
    r.high = rope->high;
    r.gain = rope->gain;
    r.original = rope->original_positions;
    launch_rope_table(r, table, rope->max_positions, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_paged_append(const chimera_paged* cache, int32_t dtype, const void* q, const void* k, const void* v,
                                    int64_t ld, int32_t n_heads, const int32_t* seq, const int32_t* pos, int32_t rows,
                                    const chimera_rope* rope, const void* table, const float* q_gain,
                                    const float* k_gain, float eps, void* q_out, int64_t ldo, void* stream) {
  return guard([&] {
    check_paged(cache);
    check_dtype(dtype);
    REQUIRE(rows >= 0 && rows <= 1 << 30, CHIMERA_EINVAL, "rows in [0, 2^30]");
    const int64_t hd = cache->head_dim;
    if (q == nullptr) {
      REQUIRE(n_heads == 0 && q_out == nullptr && q_gain == nullptr, CHIMERA_EINVAL,
              "without q, n_heads is 0 and q_out and q_gain are null");
    } else {
      check_heads(cache, n_heads);
      REQUIRE(q_out != nullptr, CHIMERA_EINVAL, "null argument");
      REQUIRE(ldo >= n_heads * hd, CHIMERA_EINVAL, "row stride below n_heads * head_dim");
      REQUIRE(q_out != q || (dtype == cache->dtype && ldo == ld), CHIMERA_EINVAL,
              "q_out may be q only with the same type and row stride");
    }
    REQUIRE(rows == 0 || (k && v && seq && pos), CHIMERA_EINVAL, "null argument");
    REQUIRE(ld >= std::max<int64_t>(n_heads, cache->n_heads) * hd, CHIMERA_EINVAL,
            "row stride below n_heads * head_dim");
    AppendArgs a{};
    if (rope != nullptr) {
      check_rope(rope);
      REQUIRE(rope->rot_dim <= hd, CHIMERA_EINVAL, "rot_dim past head_dim");
      REQUIRE(table != nullptr, CHIMERA_EINVAL, "null table");
      check_aligned(table, "table");
      a.table = (const float2*)table;
      a.pairs = rope->rot_dim / 2;
      a.cross = rope->layout == CHIMERA_ROPE_HALF;
      a.positions = rope->max_positions;
    } else {
      REQUIRE(table == nullptr, CHIMERA_EINVAL, "a table without its rope");
    }
    if (q_gain != nullptr || k_gain != nullptr)
      REQUIRE(std::isfinite(eps) && eps > 0.f, CHIMERA_EINVAL, "eps must be finite and positive");
    hipStream_t st = check_stream(stream);
    if (rows == 0) return;
    a.q = q;
    a.k = k;
    a.v = v;
    a.ld = ld;
    a.q_out = q_out;
    a.ldo = ldo;
    a.seq = seq;
    a.pos = pos;
    a.q_gain = q_gain;
    a.k_gain = k_gain;
    a.eps = eps;
    a.Hq = n_heads;
    a.rows = rows;
    launch_paged_append(dtype, cache->dtype, view(cache), a, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_paged_attn_bytes(const chimera_paged* cache, int32_t n_heads, int32_t rows, int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_attn_rows(cache, n_heads, rows);
    *bytes = paged_attn_bytes((int64_t)cache->max_pages * cache->page_size, rows, cache->batch,
                              n_heads / cache->n_heads, cache->n_heads, cache->head_dim, (int)esize(cache->dtype));
  });
}

chimera_status chimera_paged_attn(const chimera_paged* cache, const void* q, int64_t ldq, int32_t n_heads,
                                  const int32_t* row0, const int32_t* n_b, int32_t rows, int32_t window, int32_t sinks,
                                  float scale, void* out, int64_t ldo, void* ws, int64_t ws_bytes, void* stream) {
  return guard([&] {
    check_attn_rows(cache, n_heads, rows);
    REQUIRE(row0 != nullptr || rows == cache->batch, CHIMERA_EINVAL, "without row0, rows must be the batch");
    REQUIRE(rows == 0 || (q && n_b && out), CHIMERA_EINVAL, "null argument");
    REQUIRE(window >= 0 && window <= 1 << 30 && sinks >= 0 && sinks <= 1 << 30, CHIMERA_EINVAL,
            "window and sinks in [0, 2^30]");
    const int64_t es = (int64_t)esize(cache->dtype), width = (int64_t)n_heads * cache->head_dim;
    REQUIRE(ldq >= width && ldo >= width, CHIMERA_EINVAL, "row stride below n_heads * head_dim");
    REQUIRE(ldq * es % 16 == 0, CHIMERA_EINVAL, "rows of q must start at multiples of 16 bytes");
    check_aligned(q, "q");
    REQUIRE(std::isfinite(scale) && std::fabs(scale) <= 0x1p127f, CHIMERA_EINVAL,
            "scale must be finite, at most 2^127 in magnitude");  // times log2(e) it still is
    const int64_t cap = (int64_t)cache->max_pages * cache->page_size;
    const int group = n_heads / cache->n_heads;
    const int64_t need = paged_attn_bytes(cap, rows, cache->batch, group, cache->n_heads, cache->head_dim, (int)es);
    REQUIRE(need == 0 || ws != nullptr, CHIMERA_EINVAL, "null workspace");
    REQUIRE(ws_bytes >= need, CHIMERA_ENOMEM, "workspace too small");
    check_aligned(ws, "workspace");
    hipStream_t st = check_stream(stream);
    if (rows == 0) return;
    PagedAttnArgs a{};
    a.q = q;
    a.ldq = ldq;
    a.out = out;
    a.ldo = ldo;
    a.row0 = row0;
    a.n_b = n_b;
    a.rows = rows;
    a.Hq = n_heads;
    a.group = group;
    a.window = window;
    a.sinks = sinks;
    // a masked score is -inf and must weigh nothing where scale is 0 too: 2^-140 of a
    // score is no weight's last bit
    a.scale2 = std::max(std::fabs(scale) * 1.44269504088896340736f, 0x1p-140f);
    a.flip = scale < 0.f;
    launch_paged_attn(cache->dtype, view(cache), a, ws, st);
    HIPCK(hipGetLastError());
  });
}

chimera_status chimera_accept_bytes(int32_t batch, int32_t n_nodes, int32_t vocab, int32_t drawn, int64_t* bytes) {
  return guard([&] {
    REQUIRE(bytes != nullptr, CHIMERA_EINVAL, "null bytes");
    check_tree(batch, n_nodes, vocab);
    *bytes = accept_bytes(batch, n_nodes, vocab, drawn != 0);
  });
}

chimera_status chimera_accept(int32_t dtype, const void* logits, int64_t ld, const void* draft, int64_t ldd, int32_t vocab,
                              const int32_t* tokens, const int32_t* parent, int32_t n_nodes, int32_t batch,
                              float temperature, const double* u, int32_t* new_tokens, int32_t* n_new,
                              int32_t* path_nodes, void* ws, int64_t ws_bytes, void* stream) {
  return guard([&] {
    check_dtype(dtype);
    check_tree(batch, n_nodes, vocab);
    REQUIRE(logits && tokens && u && new_tokens && n_new && ws, CHIMERA_EINVAL, "null argument");
    REQUIRE(ld >= vocab && (draft == nullptr || ldd >= vocab), CHIMERA_EINVAL, "row stride below vocab");
    REQUIRE(std::isfinite(temperature) && temperature > 0.f, CHIMERA_EINVAL, "temperature must be finite and positive");
    AcceptArgs a{};
    int depth[64] = {0};
    for (int i = 0; i < n_nodes; ++i) {
      const int p = parent ? parent[i] : i - 1;
      REQUIRE(i == 0 ? p == -1 : (p >= 0 && p < i), CHIMERA_EINVAL,
              "node 0 must be the root and a parent must precede its child");
      REQUIRE(draft == nullptr || p == i - 1, CHIMERA_EINVAL, "tokens drawn from a draft form a chain");
      depth[i] = i == 0 ? 0 : depth[p] + 1;
      a.K = std::max(a.K, depth[i]);
      a.tree.set(i, p);
      if (i > 0) a.inner |= (uint64_t)1 << p;
    }
    check_aligned(ws, "workspace");
    REQUIRE(ws_bytes >= accept_bytes(batch, n_nodes, vocab, draft != nullptr), CHIMERA_ENOMEM, "workspace too small");
    hipStream_t st = check_stream(stream);
    a.logits = logits;
    a.ld = ld;
    a.draft = draft;
    a.ldd = ldd;
    a.tokens = tokens;
    a.u = u;
    a.B = batch;
    a.N = n_nodes;
    a.V = vocab;
    a.scale = accept_scale(temperature);
    a.new_tokens = new_tokens;
    a.n_new = n_new;
    a.path = path_nodes;
    a.none = -1;
    accept_carve(a, ws);
    launch_accept(dtype, a, st);
    HIPCK(hipGetLastError());
  });
}

}  // extern "C"
