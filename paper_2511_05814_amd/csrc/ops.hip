// C entries of the attention half of a layer and of drafted tokens: argument
// checks and launches.
#include <algorithm>

#include "common.hpp"
#include "moe_offload.h"

using namespace moe;

namespace {

bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }

// a * b * c for non-negative factors, or -1 past 2^62
int64_t product(int64_t a, int64_t b, int64_t c = 1) {
  int64_t v;
  if (__builtin_mul_overflow(a, b, &v) || __builtin_mul_overflow(v, c, &v) || v >= (int64_t)1 << 62) return -1;
  return v;
}

int check_dtype(int dtype) {
  if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return fail(MOE_ERR_ARG, "dtype must be MOE_DTYPE_F32 or MOE_DTYPE_BF16");
  return MOE_OK;
}

// A row-strided operand: rows of `width` elements of `bytes` bytes, aligned to
// `align`, and non-NULL (a tensor without elements has no address) if there are rows.
int check_rows(const char *name, const void *p, int64_t stride, int64_t width, int bytes, int align, int rows) {
  if ((!p && rows) || misaligned(p, align)) return fail(MOE_ERR_ARG, "%s must be a non-NULL device pointer aligned to %d bytes", name, align);
  if (stride < width || stride > (int64_t)1 << 40) return fail(MOE_ERR_ARG, "%s: a stride of %lld for rows of %lld", name, (long long)stride, (long long)width);
  if (stride * bytes % align) return fail(MOE_ERR_ARG, "%s: its stride must be a multiple of %d bytes", name, align);
  return MOE_OK;
}

int element(int dtype) { return dtype == MOE_DTYPE_F32 ? 4 : 2; }

int launched(hipError_t e, const char *what) {
  return e == hipSuccess ? MOE_OK : fail(MOE_ERR_HIP, "%s failed: %s", what, hipGetErrorString(e));
}

// `rows` stretches of memory of `width` bytes each, `stride` bytes apart.
struct Span {
  const void *at;
  int64_t stride, width, rows;
};
Span rows_of(const void *p, int64_t stride, int64_t width, int bytes, int64_t rows) { return Span{p, stride * bytes, width * bytes, rows}; }
Span block_of(const void *p, int64_t bytes) { return Span{p, bytes, bytes, 1}; }
Span pool_of(const moe_kv4_batch *b) {
  return rows_of(b->pool, (int64_t)b->kv_heads * b->page_size * b->head_dim * 9 / 8, (int64_t)b->kv_heads * b->page_size * b->head_dim * 9 / 8, 1, b->pages);
}

// Whether two spans share a byte: row i of a begins at i a.stride, row j of b at
// d + j b.stride.
bool share(const Span &a, const Span &b) {
  typedef __int128 Wide;
  if (!a.at || !b.at || a.rows < 1 || b.rows < 1) return false;
  const Wide d = (Wide)(uintptr_t)b.at - (Wide)(uintptr_t)a.at;
  if (d >= (Wide)a.stride * (a.rows - 1) + a.width || d + (Wide)b.stride * (b.rows - 1) + b.width <= 0) return false;
  if (a.rows > b.rows) return share(b, a);
  auto floor_div = [](Wide x, Wide y) { return x / y - (x % y < 0 ? 1 : 0); };
  if (a.stride == b.stride) {
    // rows are no wider than the stride: row j of b can meet rows j + k and j + k + 1 of a
    const Wide k = floor_div(d, a.stride), rest = d - k * a.stride;
    return (rest < a.width && k < a.rows && -k < b.rows) || (rest + b.width > a.stride && k + 1 < a.rows && -k - 1 < b.rows);
  }
  for (int64_t i = 0; i < a.rows; ++i) {
    // the first row of b that ends after row i's start, the last that begins before its end
    const Wide start = (Wide)a.stride * i - d;
    const Wide first = floor_div(start - b.width, b.stride) + 1, last = floor_div(start + a.width - 1, b.stride);
    if ((first < 0 ? 0 : first) <= (last < b.rows ? last : b.rows - 1)) return true;
  }
  return false;
}
bool exactly(const Span &a, const Span &b) {
  return a.at == b.at && a.width == b.width && a.rows == b.rows && (a.rows == 1 || a.stride == b.stride);
}

// What is written may not overlap what other threads of the launch read, unless
// `in_place`: each element is then read before its own thread writes it.
int check_apart(const char *out, const Span &o, const char *in, const Span &i, bool in_place = false) {
  if (!share(o, i) || (in_place && exactly(o, i))) return MOE_OK;
  return fail(MOE_ERR_ARG, "%s overlaps %s", out, in);
}

int check_batch(const moe_kv4_batch *b) {
  if (!b) return fail(MOE_ERR_ARG, "NULL batch");
  if (b->head_dim != 64 && b->head_dim != 128) return fail(MOE_ERR_ARG, "head_dim must be 64 or 128, not %d", b->head_dim);
  if (b->page_size < 16 || b->page_size > 1024 || (b->page_size & (b->page_size - 1)))
    return fail(MOE_ERR_ARG, "page_size must be a power of two in [16, 1024], not %d", b->page_size);
  if (b->kv_heads < 1 || b->kv_heads > 1024) return fail(MOE_ERR_ARG, "kv_heads must be in [1, 1024]");
  if (b->pages < 1) return fail(MOE_ERR_ARG, "pages must be >= 1");
  if (b->table_cols < 1 || product(b->table_cols, b->page_size) > (int64_t)1 << 30)
    return fail(MOE_ERR_ARG, "table_cols must be in [1, 2^30 / page_size]");
  if (b->table_stride < b->table_cols) return fail(MOE_ERR_ARG, "table_stride < table_cols");
  if (b->seqs < 1 || b->seqs > 1 << 20) return fail(MOE_ERR_ARG, "seqs must be in [1, 2^20]");
  if (b->tokens < 0 || b->tokens > 1 << 24) return fail(MOE_ERR_ARG, "tokens must be in [0, 2^24]");
  if (!b->pool || misaligned(b->pool, 16)) return fail(MOE_ERR_ARG, "pool must be a non-NULL 16-byte aligned device pointer");
  if (!b->page_table || !b->q_start || !b->kv_len || misaligned(b->page_table, 4) || misaligned(b->q_start, 4) || misaligned(b->kv_len, 4))
    return fail(MOE_ERR_ARG, "page_table, q_start and kv_len must be non-NULL device arrays of int32");
  return MOE_OK;
}

KvAttnShape tree_shape(const moe_kv4_batch *b, int heads, int dtype, int max_new, int max_len) {
  return kv4_tree_shape(b->seqs, b->kv_heads, heads, b->tokens, max_new, max_len, (int64_t)b->table_cols * b->page_size, b->head_dim,
                        dtype == MOE_DTYPE_F32);
}

// Rows that a launch of attention leaves to be joined: of every split, or two
// places of each of the tree kernel's workgroups.
size_t parts_rows(const KvAttnShape &s, const moe_kv4_batch *b, int heads) {
  return s.splits == 1 ? 0 : s.tiles ? (size_t)s.splits * 2 * 16 * s.tiles : (size_t)s.splits * b->tokens * heads;
}
size_t parts_bytes(const KvAttnShape &s, const moe_kv4_batch *b, int heads) {
  const size_t rows = parts_rows(s, b, heads);
  return rows * (b->head_dim + 2) * sizeof(float) + (s.tiles && rows ? ((size_t)b->seqs + 1) * sizeof(int32_t) : 0);
}

int check_heads(const moe_kv4_batch *b, int heads) {
  if (heads < 1 || heads > 4096 || heads % b->kv_heads)
    return fail(MOE_ERR_ARG, "heads (%d) must be a multiple of kv_heads (%d), at most 4096", heads, b->kv_heads);
  return MOE_OK;
}

Kv4 kv_of(const moe_kv4_batch *b) {
  Kv4 k;
  k.pool = static_cast<uint8_t *>(b->pool);
  k.page_table = b->page_table;
  k.q_start = b->q_start;
  k.kv_len = b->kv_len;
  k.table_stride = b->table_stride;
  k.pages = b->pages;
  k.page_log2 = __builtin_ctz((unsigned)b->page_size);
  k.kv_heads = b->kv_heads;
  k.table_cols = b->table_cols;
  k.seqs = b->seqs;
  k.tokens = b->tokens;
  return k;
}

int check_tree(const int32_t *q_start, int seqs, int tokens) {
  if (seqs < 1 || seqs > 1 << 20) return fail(MOE_ERR_ARG, "seqs must be in [1, 2^20]");
  if (tokens < 0 || tokens > 1 << 24) return fail(MOE_ERR_ARG, "tokens must be in [0, 2^24]");
  if (!q_start || misaligned(q_start, 4)) return fail(MOE_ERR_ARG, "q_start must be a non-NULL device array of int32");
  return MOE_OK;
}

// An array of 4-byte elements, non-NULL if it has any.
int check_ints(const char *name, const void *p, int n) {
  if ((!p && n) || misaligned(p, 4)) return fail(MOE_ERR_ARG, "%s must be a non-NULL device pointer aligned to 4 bytes", name);
  return MOE_OK;
}

#define CHECK(expr)                    \
  do {                                 \
    const int rc_ = (expr);            \
    if (rc_ != MOE_OK) return rc_;     \
  } while (0)

}  // namespace

extern "C" {

size_t moe_q4_matrix_bytes(size_t n, size_t k) {
  if (n < 1 || k < 64 || k % 64 || n > ((size_t)1 << 40) / k) return 0;
  return n * (k / 2) + n * (k / 64) * 3;
}

int moe_q4_matmul(const void *x, int64_t x_stride, const void *w, void *y, int64_t y_stride, int rows, int n, int k,
                  int dtype, void *stream) {
  CHECK(check_dtype(dtype));
  if (rows < 0 || rows > 1 << 20) return fail(MOE_ERR_ARG, "rows must be in [0, 2^20]");
  if (n < 1 || n > 1 << 24) return fail(MOE_ERR_ARG, "n must be in [1, 2^24]");
  if (k < 64 || k % 64 || k > 1 << 20) return fail(MOE_ERR_ARG, "k must be a multiple of 64 in [64, 2^20]");
  if (q4_groups(rows, n) > kMaxGroups) return fail(MOE_ERR_ARG, "too many rows times n");
  if (!w || misaligned(w, 16)) return fail(MOE_ERR_ARG, "w must be a non-NULL 16-byte aligned device pointer");
  CHECK(check_rows("x", x, x_stride, k, element(dtype), 16, rows));
  CHECK(check_rows("y", y, y_stride, n, element(dtype), element(dtype), rows));
  if (rows == 0) return MOE_OK;
  const Span to = rows_of(y, y_stride, n, element(dtype), rows);
  CHECK(check_apart("y", to, "x", rows_of(x, x_stride, k, element(dtype), rows)));
  CHECK(check_apart("y", to, "w", block_of(w, (int64_t)moe_q4_matrix_bytes(n, k))));
  Q4Args a;
  a.x = x;
  a.y = y;
  a.codes = static_cast<const uint8_t *>(w);
  a.scales = a.codes + (size_t)n * (k / 2);
  a.zeros = a.scales + (size_t)n * (k / 64) * 2;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.rows = rows;
  a.n = n;
  a.k = k;
  return launched(launch_q4_matmul(a, dtype == MOE_DTYPE_F32, static_cast<hipStream_t>(stream)), "4-bit product");
}

int moe_kv4_append(const moe_kv4_batch *b, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                   const void *v, int64_t v_stride, const float *cos, const float *sin, int max_pos, int rot_dim,
                   void *q_out, int64_t q_out_stride, int heads, int dtype, void *stream) {
  return moe_kv4_append_at(b, nullptr, q, q_stride, k, k_stride, v, v_stride, cos, sin, max_pos, rot_dim, q_out, q_out_stride, heads,
                           dtype, stream);
}

int moe_kv4_append_at(const moe_kv4_batch *b, const int32_t *pos, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                      const void *v, int64_t v_stride, const float *cos, const float *sin, int max_pos, int rot_dim,
                      void *q_out, int64_t q_out_stride, int heads, int dtype, void *stream) {
  CHECK(check_batch(b));
  if (misaligned(pos, 4)) return fail(MOE_ERR_ARG, "pos must be a device array of int32");
  CHECK(check_dtype(dtype));
  CHECK(check_heads(b, heads));
  const int bytes = element(dtype), d = b->head_dim;
  CHECK(check_rows("q", q, q_stride, (int64_t)heads * d, bytes, 16, b->tokens));
  CHECK(check_rows("k", k, k_stride, (int64_t)b->kv_heads * d, bytes, 16, b->tokens));
  CHECK(check_rows("v", v, v_stride, (int64_t)b->kv_heads * d, bytes, 16, b->tokens));
  CHECK(check_rows("q_out", q_out, q_out_stride, (int64_t)heads * d, bytes, 16, b->tokens));
  if (rot_dim < 0 || rot_dim > d || rot_dim % 16) return fail(MOE_ERR_ARG, "rot_dim must be a multiple of 16 in [0, head_dim], not %d", rot_dim);
  if (max_pos < 1) return fail(MOE_ERR_ARG, "max_pos must be >= 1");
  if (rot_dim && (!cos || !sin || misaligned(cos, 16) || misaligned(sin, 16)))
    return fail(MOE_ERR_ARG, "cos and sin must be non-NULL 16-byte aligned device pointers");
  if (product(b->tokens, heads + 2 * b->kv_heads, d / 8) > kMaxGroups * 256) return fail(MOE_ERR_ARG, "too many tokens times heads");
  if (b->tokens == 0) return MOE_OK;
  const Span to = rows_of(q_out, q_out_stride, (int64_t)heads * d, bytes, b->tokens), pool = pool_of(b);
  const Span qs = rows_of(q, q_stride, (int64_t)heads * d, bytes, b->tokens);
  const Span ks = rows_of(k, k_stride, (int64_t)b->kv_heads * d, bytes, b->tokens), vs = rows_of(v, v_stride, (int64_t)b->kv_heads * d, bytes, b->tokens);
  CHECK(check_apart("q_out", to, "q (it may be q itself without rotation)", qs, rot_dim == 0));
  CHECK(check_apart("q_out", to, "k", ks));
  CHECK(check_apart("q_out", to, "v", vs));
  CHECK(check_apart("q_out", to, "the cache", pool));
  CHECK(check_apart("the cache", pool, "q", qs));
  CHECK(check_apart("the cache", pool, "k", ks));
  CHECK(check_apart("the cache", pool, "v", vs));
  if (pos) {
    CHECK(check_apart("q_out", to, "pos", block_of(pos, (int64_t)b->tokens * 4)));
    CHECK(check_apart("the cache", pool, "pos", block_of(pos, (int64_t)b->tokens * 4)));
  }
  if (rot_dim) {
    const Span c = block_of(cos, (int64_t)max_pos * rot_dim * 2), n = block_of(sin, (int64_t)max_pos * rot_dim * 2);
    CHECK(check_apart("q_out", to, "cos", c));
    CHECK(check_apart("q_out", to, "sin", n));
    CHECK(check_apart("the cache", pool, "cos", c));
    CHECK(check_apart("the cache", pool, "sin", n));
  }
  KvAppendArgs a;
  a.kv = kv_of(b);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.cos = cos;
  a.sin = sin;
  a.pos = pos;
  a.max_pos = max_pos;
  a.rot = rot_dim;
  a.heads = heads;
  return launched(launch_kv4_append(a, d, dtype == MOE_DTYPE_F32, static_cast<hipStream_t>(stream)), "cache append");
}

int moe_kv4_read(const moe_kv4_batch *b, void *k, void *v, int dtype, void *stream) {
  CHECK(check_batch(b));
  CHECK(check_dtype(dtype));
  if ((b->tokens && (!k || !v)) || misaligned(k, 16) || misaligned(v, 16)) return fail(MOE_ERR_ARG, "k and v must be non-NULL 16-byte aligned device pointers");
  if (product(b->tokens, 2 * b->kv_heads, b->head_dim / 8) > kMaxGroups * 256) return fail(MOE_ERR_ARG, "too many tokens times heads");
  if (b->tokens == 0) return MOE_OK;
  const int64_t size = (int64_t)b->tokens * b->kv_heads * b->head_dim * element(dtype);
  CHECK(check_apart("k", block_of(k, size), "v", block_of(v, size)));
  CHECK(check_apart("k", block_of(k, size), "the cache", pool_of(b)));
  CHECK(check_apart("v", block_of(v, size), "the cache", pool_of(b)));
  KvReadArgs a;
  a.kv = kv_of(b);
  a.k = k;
  a.v = v;
  return launched(launch_kv4_read(a, b->head_dim, dtype == MOE_DTYPE_F32, static_cast<hipStream_t>(stream)), "cache read");
}

size_t moe_kv4_attention_workspace_bytes(const moe_kv4_batch *b, int heads, int max_new, int max_len) {
  if (check_batch(b) != MOE_OK || check_heads(b, heads) != MOE_OK || max_new < 1 || max_len < 1) return 0;
  if (product(b->seqs, b->kv_heads) > kMaxGroups || product(b->tokens, heads) > (int64_t)1 << 30) return 0;
  return parts_bytes(kv4_attention_shape(b->seqs, b->kv_heads, heads, b->tokens, max_new, max_len), b, heads);
}

size_t moe_kv4_tree_attention_workspace_bytes(const moe_kv4_batch *b, int heads, int dtype, int max_new, int max_len) {
  if (check_dtype(dtype) != MOE_OK || check_batch(b) != MOE_OK || check_heads(b, heads) != MOE_OK || max_new < 1 || max_len < 1) return 0;
  if (product(b->seqs, b->kv_heads) > kMaxGroups || product(b->tokens, heads) > (int64_t)1 << 30) return 0;
  return parts_bytes(tree_shape(b, heads, dtype, max_new, max_len), b, heads);
}

}  // extern "C"

namespace {

// Both attentions; `seen` is NULL where tokens see what is before them.
int attention(const moe_kv4_batch *b, const void *q, int64_t q_stride, const uint32_t *seen, int words, void *o, int64_t o_stride,
              int heads, float scale, int dtype, int max_new, int max_len, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_batch(b));
  CHECK(check_dtype(dtype));
  CHECK(check_heads(b, heads));
  const int bytes = element(dtype), d = b->head_dim;
  CHECK(check_rows("q", q, q_stride, (int64_t)heads * d, bytes, 16, b->tokens));
  CHECK(check_rows("o", o, o_stride, (int64_t)heads * d, bytes, 16, b->tokens));
  if (max_new < 1 || max_len < 1) return fail(MOE_ERR_ARG, "max_new and max_len must be >= 1");
  if (product(b->seqs, b->kv_heads) > kMaxGroups || product(b->tokens, heads) > (int64_t)1 << 30)
    return fail(MOE_ERR_ARG, "sequences times kv_heads must be below 2^24 and tokens times heads at most 2^30");
  KvAttnArgs a;
  a.kv = kv_of(b);
  a.q = q;
  a.o = o;
  a.q_stride = q_stride;
  a.o_stride = o_stride;
  a.scale = scale;
  a.heads = heads;
  const KvAttnShape shape = seen ? tree_shape(b, heads, dtype, max_new, max_len)
                                 : kv4_attention_shape(b->seqs, b->kv_heads, heads, b->tokens, max_new, max_len);
  a.splits = shape.splits;
  a.row_blocks = shape.row_blocks;
  a.prompt = shape.prompt;
  const size_t rows = parts_rows(shape, b, heads), need = parts_bytes(shape, b, heads);
  if (workspace_bytes < need || (need && (!workspace || misaligned(workspace, 16))))
    return fail(MOE_ERR_ARG, "workspace must be 16-byte aligned and hold %zu bytes (got %zu)", need, workspace_bytes);
  if (b->tokens == 0) return MOE_OK;
  const Span to = rows_of(o, o_stride, (int64_t)heads * d, bytes, b->tokens), qs = rows_of(q, q_stride, (int64_t)heads * d, bytes, b->tokens);
  CHECK(check_apart("o", to, "q", qs, true));
  CHECK(check_apart("o", to, "the cache", pool_of(b)));
  const Span bits = block_of(seen, (int64_t)b->tokens * words * 4);
  CHECK(check_apart("o", to, "seen", bits));
  if (need) {
    CHECK(check_apart("the workspace", block_of(workspace, (int64_t)need), "seen", bits));
    CHECK(check_apart("the workspace", block_of(workspace, (int64_t)need), "q", qs));
    CHECK(check_apart("the workspace", block_of(workspace, (int64_t)need), "o", to));
    CHECK(check_apart("the workspace", block_of(workspace, (int64_t)need), "the cache", pool_of(b)));
  }
  a.part = static_cast<float *>(workspace);
  a.ml = a.part ? a.part + rows * d : nullptr;
  a.plan = a.part ? reinterpret_cast<int32_t *>(a.ml + 2 * rows) : nullptr;
  a.seen = seen;
  a.words = words;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f32 = dtype == MOE_DTYPE_F32;
  return launched(shape.tiles ? launch_kv4_tree(a, shape.tiles, d, f32, s) : launch_kv4_attention(a, d, f32, s), "cache attention");
}

}  // namespace

extern "C" {

int moe_kv4_attention(const moe_kv4_batch *b, const void *q, int64_t q_stride, void *o, int64_t o_stride, int heads,
                      float scale, int dtype, int max_new, int max_len, void *workspace, size_t workspace_bytes,
                      void *stream) {
  return attention(b, q, q_stride, nullptr, 0, o, o_stride, heads, scale, dtype, max_new, max_len, workspace, workspace_bytes, stream);
}

int moe_kv4_tree_attention(const moe_kv4_batch *b, const void *q, int64_t q_stride, const uint32_t *seen, int words, void *o,
                           int64_t o_stride, int heads, float scale, int dtype, int max_new, int max_len, void *workspace,
                           size_t workspace_bytes, void *stream) {
  if (words < 1 || words > kMaxTree / 32) return fail(MOE_ERR_ARG, "words must be in [1, %d], not %d", kMaxTree / 32, words);
  if (!seen || misaligned(seen, 4)) return fail(MOE_ERR_ARG, "seen must be a non-NULL device array of uint32");
  return attention(b, q, q_stride, seen, words, o, o_stride, heads, scale, dtype, max_new, max_len, workspace, workspace_bytes, stream);
}

int moe_kv4_keep(const moe_kv4_batch *b, void *const *pools, int n_pools, const int32_t *path, const int32_t *count, void *stream) {
  constexpr int kMost = 1024;
  if (!b || !pools || n_pools < 1 || n_pools > kMost) return fail(MOE_ERR_ARG, "NULL batch or pools, or not 1 .. %d of them", kMost);
  uintptr_t at[kMost];
  moe_kv4_batch each = *b;
  for (int i = 0; i < n_pools; ++i) {
    each.pool = pools[i];
    CHECK(check_batch(&each));
    CHECK(check_apart("a cache", pool_of(&each), "path", block_of(path, (int64_t)b->tokens * 4)));
    CHECK(check_apart("a cache", pool_of(&each), "count", block_of(count, (int64_t)b->seqs * 4)));
    at[i] = reinterpret_cast<uintptr_t>(pools[i]);
  }
  CHECK(check_ints("path", path, b->tokens));
  CHECK(check_ints("count", count, b->tokens));
  if (b->tokens == 0) return MOE_OK;
  // one cache twice would move its entries twice at once
  std::sort(at, at + n_pools);
  const uintptr_t bytes = (uintptr_t)pool_of(&each).stride * (uintptr_t)b->pages;
  for (int i = 1; i < n_pools; ++i)
    if (at[i] - at[i - 1] < bytes) return fail(MOE_ERR_ARG, "two caches overlap");
  KvKeepArgs a;
  a.path = path;
  a.count = count;
  for (int i = 0; i < n_pools; i += kKeepPools) {
    const int n = std::min(kKeepPools, n_pools - i);
    a.kv = kv_of(&each);
    for (int j = 0; j < kKeepPools; ++j) a.pools[j] = static_cast<uint8_t *>(pools[i + std::min(j, n - 1)]);
    CHECK(launched(launch_kv4_keep(a, n, b->head_dim, static_cast<hipStream_t>(stream)), "keeping cache entries"));
  }
  return MOE_OK;
}

int moe_draft_tree(const int32_t *parent, const int32_t *q_start, const int32_t *kv_len, int seqs, int tokens, int words,
                   int32_t *pos, uint32_t *seen, void *stream) {
  CHECK(check_tree(q_start, seqs, tokens));
  if (words < 1 || words > kMaxTree / 32) return fail(MOE_ERR_ARG, "words must be in [1, %d], not %d", kMaxTree / 32, words);
  CHECK(check_ints("parent", parent, tokens));
  CHECK(check_ints("kv_len", kv_len, 1));
  CHECK(check_ints("pos", pos, tokens));
  CHECK(check_ints("seen", seen, tokens));
  if (tokens == 0) return MOE_OK;
  const Span outs[2] = {block_of(pos, (int64_t)tokens * 4), block_of(seen, (int64_t)tokens * words * 4)};
  CHECK(check_apart("pos", outs[0], "seen", outs[1]));
  for (int i = 0; i < 2; ++i) {
    CHECK(check_apart(i ? "seen" : "pos", outs[i], "parent", block_of(parent, (int64_t)tokens * 4)));
    CHECK(check_apart(i ? "seen" : "pos", outs[i], "q_start", block_of(q_start, (int64_t)(seqs + 1) * 4)));
    CHECK(check_apart(i ? "seen" : "pos", outs[i], "kv_len", block_of(kv_len, (int64_t)seqs * 4)));
  }
  DraftTreeArgs a;
  a.parent = parent;
  a.q_start = q_start;
  a.kv_len = kv_len;
  a.pos = pos;
  a.seen = seen;
  a.seqs = seqs;
  a.tokens = tokens;
  a.words = words;
  return launched(launch_draft_tree(a, static_cast<hipStream_t>(stream)), "plan of a tree");
}

size_t moe_verify_drafts_workspace_bytes(int seqs, int vocab) {
  if (seqs < 1 || seqs > 1 << 20 || vocab < 1 || vocab > 1 << 24) return 0;
  const int clusters = verify_clusters(seqs, vocab);
  return clusters == 1 ? 0 : (size_t)seqs * kVerifyPasses * clusters * sizeof(uint64_t);
}

int moe_verify_drafts(const void *p, int64_t p_stride, const void *q, int64_t q_stride, const int32_t *ids, const int32_t *parent,
                      const float *u, const int32_t *q_start, int seqs, int tokens, int vocab, int dtype, int32_t *path,
                      int32_t *count, int32_t *next, void *workspace, size_t workspace_bytes, void *stream) {
  CHECK(check_dtype(dtype));
  CHECK(check_tree(q_start, seqs, tokens));
  if (vocab < 1 || vocab > 1 << 24) return fail(MOE_ERR_ARG, "vocab must be in [1, 2^24]");
  const int bytes = element(dtype);
  CHECK(check_rows("p", p, p_stride, vocab, bytes, bytes, tokens));
  if (q) CHECK(check_rows("q", q, q_stride, vocab, bytes, bytes, tokens));
  CHECK(check_ints("ids", ids, tokens));
  CHECK(check_ints("parent", parent, tokens));
  CHECK(check_ints("u", u, tokens));
  CHECK(check_ints("path", path, tokens));
  CHECK(check_ints("count", count, 1));
  CHECK(check_ints("next", next, 1));
  const size_t need = moe_verify_drafts_workspace_bytes(seqs, vocab);
  if (workspace_bytes < need || (need && (!workspace || misaligned(workspace, 16))))
    return fail(MOE_ERR_ARG, "workspace must be 16-byte aligned and hold %zu bytes (got %zu)", need, workspace_bytes);
  const Span outs[4] = {block_of(path, (int64_t)tokens * 4), block_of(count, (int64_t)seqs * 4), block_of(next, (int64_t)seqs * 4),
                        block_of(workspace, (int64_t)need)};
  const char *const names[4] = {"path", "count", "next", "the workspace"};
  for (int i = 0; i < 4; ++i) {
    for (int j = i + 1; j < 4; ++j) CHECK(check_apart(names[i], outs[i], names[j], outs[j]));
    CHECK(check_apart(names[i], outs[i], "p", rows_of(p, p_stride, vocab, bytes, tokens)));
    CHECK(check_apart(names[i], outs[i], "q", rows_of(q, q_stride, vocab, bytes, tokens)));
    CHECK(check_apart(names[i], outs[i], "ids", block_of(ids, (int64_t)tokens * 4)));
    CHECK(check_apart(names[i], outs[i], "parent", block_of(parent, (int64_t)tokens * 4)));
    CHECK(check_apart(names[i], outs[i], "u", block_of(u, (int64_t)tokens * 4)));
    CHECK(check_apart(names[i], outs[i], "q_start", block_of(q_start, (int64_t)(seqs + 1) * 4)));
  }
  VerifyArgs a;
  a.p = p;
  a.q = q;
  a.p_stride = p_stride;
  a.q_stride = q_stride;
  a.ids = ids;
  a.parent = parent;
  a.u = u;
  a.q_start = q_start;
  a.path = path;
  a.count = count;
  a.next = next;
  a.seqs = seqs;
  a.tokens = tokens;
  a.vocab = vocab;
  a.clusters = verify_clusters(seqs, vocab);
  a.slots = static_cast<uint64_t *>(workspace);
  return launched(launch_verify_drafts(a, dtype == MOE_DTYPE_F32, static_cast<hipStream_t>(stream)), "verification");
}

int moe_norm_residual(const float *h, int64_t h_stride, const void *y, int64_t y_stride, const float *gate,
                      int64_t gate_stride, const float *post, const float *pre, float residual_scale, float eps,
                      float *h_out, int64_t h_out_stride, void *x_out, int64_t x_stride, int rows, int d, int dtype,
                      void *stream) {
  CHECK(check_dtype(dtype));
  if (rows < 0 || rows > 1 << 24) return fail(MOE_ERR_ARG, "rows must be in [0, 2^24]");
  if (d < 8 || d % 8 || d > 16384) return fail(MOE_ERR_ARG, "d must be a multiple of 8 in [8, 16384]");
  if (norm_groups(rows, d) > kMaxGroups) return fail(MOE_ERR_ARG, "rows of more than %d channels must be fewer than 2^24", kNormNarrow);
  const int bytes = element(dtype);
  CHECK(check_rows("h", h, h_stride, d, 4, 16, rows));
  if (y) CHECK(check_rows("y", y, y_stride, d, bytes, 16, rows));
  if (!y && rows && (gate || post)) return fail(MOE_ERR_ARG, "gate and post need y");
  if (gate && gate_stride) CHECK(check_rows("gate", gate, gate_stride, d, 4, 16, rows));
  if (misaligned(gate, 16) || misaligned(post, 16) || misaligned(pre, 16)) return fail(MOE_ERR_ARG, "gate, post and pre must be 16-byte aligned");
  if (!h_out && !x_out && rows) return fail(MOE_ERR_ARG, "neither h_out nor x_out is wanted");
  if (h_out) CHECK(check_rows("h_out", h_out, h_out_stride, d, 4, 16, rows));
  if (x_out) CHECK(check_rows("x_out", x_out, x_stride, d, bytes, 16, rows));
  if (rows == 0) return MOE_OK;
  // A thread reads its channels of h, y, gate and post, writes h_out, reads pre and writes x_out.
  const Span to_h = rows_of(h_out, h_out_stride, d, 4, rows), to_x = rows_of(x_out, x_stride, d, bytes, rows);
  const Span hs = rows_of(h, h_stride, d, 4, rows), ys = rows_of(y, y_stride, d, bytes, rows);
  const Span gs = rows_of(gate, gate_stride ? gate_stride : d, d, 4, gate_stride ? rows : 1);
  const Span posts = rows_of(post, d, d, 4, 1), pres = rows_of(pre, d, d, 4, 1);
  CHECK(check_apart("h_out", to_h, "h (it may be h itself)", hs, true));
  CHECK(check_apart("h_out", to_h, "y", ys, true));
  CHECK(check_apart("h_out", to_h, "gate", gs, true));
  CHECK(check_apart("h_out", to_h, "post", posts, true));
  CHECK(check_apart("h_out", to_h, "pre", pres));
  CHECK(check_apart("h_out", to_h, "x_out", to_x));
  CHECK(check_apart("x_out", to_x, "h", hs, true));
  CHECK(check_apart("x_out", to_x, "y (it may be y itself)", ys, true));
  CHECK(check_apart("x_out", to_x, "gate", gs, true));
  CHECK(check_apart("x_out", to_x, "post", posts, true));
  CHECK(check_apart("x_out", to_x, "pre", pres, true));
  NormArgs a;
  a.h = h;
  a.gate = gate;
  a.post = post;
  a.pre = pre;
  a.y = y;
  a.h_out = h_out;
  a.x_out = x_out;
  a.h_stride = h_stride;
  a.y_stride = y_stride;
  a.gate_stride = gate_stride;
  a.h_out_stride = h_out_stride;
  a.x_stride = x_stride;
  a.residual_scale = residual_scale;
  a.eps = eps;
  a.rows = rows;
  a.d = d;
  return launched(launch_norm_residual(a, dtype == MOE_DTYPE_F32, static_cast<hipStream_t>(stream)), "norm");
}

}  // extern "C"
