// gm_ops.cpp -- host side of the operators on caller tensors: argument checks,
// then one launch function each (gm_ops.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "gm.h"
#include "gm_error.h"
#include "gm_ops.h"

using namespace gm;

namespace {

constexpr int64_t kPositions = int64_t(1) << 24;   // positions are exact in fp32 below this

bool misaligned(const void* p, unsigned to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

int check_dtype(int dtype) {
  return dtype < GM_DTYPE_F32 || dtype > GM_DTYPE_F16 ? inval("bad dtype") : GM_OK;
}

int check_head_dim(int hd) {
  return hd != 32 && hd != 64 && hd != 128 ? inval("head_dim must be 32, 64 or 128") : GM_OK;
}

// A [B, n, H, hd] tensor; no element is looked at if one of B, n, H is 0.
int check_tensor(const gm_tensor& t, int dtype, int64_t B, int64_t n, int64_t H, int hd, bool output) {
  if (B == 0 || n == 0 || H == 0) return GM_OK;
  if (!t.p) return inval("a tensor pointer is NULL");
  const int64_t esz = dtype == GM_DTYPE_F32 ? 4 : 2;
  if (misaligned(t.p, 16)) return inval("tensors must be 16-byte aligned");
  const int64_t len[3] = {B, n, H}, stride[3] = {t.batch, t.token, t.head};
  for (int i = 0; i < 3; ++i) {
    if (len[i] == 1) continue;
    if (stride[i] < 0) return inval("tensor strides may not be negative");
    if (stride[i] >= (int64_t(1) << 48)) return inval("a tensor stride is out of range");
    if (stride[i] * esz % 16) return inval("tensor strides must be multiples of 16 bytes");
    if (output && stride[i] < hd) return inval("an output tensor's elements overlap");
  }
  if (output) {
    // dimensions by stride: each must step over all of the smaller ones
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j + 1 < 3; ++j)
        if (stride[order[j]] > stride[order[j + 1]]) {
          const int o = order[j];
          order[j] = order[j + 1];
          order[j + 1] = o;
        }
    int64_t span = hd;
    for (int i = 0; i < 3; ++i) {
      if (len[order[i]] == 1) continue;
      if (stride[order[i]] < span) return inval("an output tensor's elements overlap");
      span += stride[order[i]] * (len[order[i]] - 1);
    }
  }
  return GM_OK;
}

int check_cache(const gm_kv_cache* c) {
  if (!c) return inval("cache is NULL");
  if (c->bits != 8 && c->bits != 4) return inval("cache bits must be 8 or 4");
  if (int rc = check_head_dim(c->head_dim)) return rc;
  if (c->batch < 1 || c->heads < 1 || c->batch > (1 << 20) || c->heads > (1 << 16))
    return inval("cache batch and heads must be positive");
  if (c->max_seq < 64 || c->max_seq % 64) return inval("cache max_seq must be a multiple of 64");
  if (c->max_seq >= kPositions) return inval("cache max_seq must be below 2^24");
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return inval("a cache pointer is NULL");
  if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->k_scale, 16) ||
      misaligned(c->v_scale, 16) || misaligned(c->valid, 8))
    return inval("cache memory must be 16-byte aligned (valid: 8)");
  return GM_OK;
}

int check_rows(const gm_kv_cache* c, int dtype, int B, int n, const gm_tensor& k, const gm_tensor& v,
               const int32_t* start, const int32_t* count, const int32_t* mask, bool output) {
  int rc = check_cache(c);
  if (rc || (rc = check_dtype(dtype))) return rc;
  if (B < 0 || B > c->batch) return inval("B must be at most the cache's batch");
  if (n < 0 || n >= kPositions) return inval("n must be below 2^24");
  if ((rc = check_tensor(k, dtype, B, n, c->heads, c->head_dim, output)) ||
      (rc = check_tensor(v, dtype, B, n, c->heads, c->head_dim, output)))
    return rc;
  if (misaligned(start, 4) || misaligned(count, 4) || misaligned(mask, 4))
    return inval("int32 arrays must be 4-byte aligned");
  // a launch has fewer than 2^32 threads, 8 channels each
  if (static_cast<double>(B) * n * c->heads * 2 * (c->head_dim / 8) >= 4294967040.0)
    return inval("B * n * heads * head_dim / 4 must be below 2^32 - 256");
  return GM_OK;
}

int check_scores(const gm_scores& s) {
  if (!(s.scale > 0.f) || !std::isfinite(s.scale)) return inval("scale must be positive and finite");
  if (s.softcap != 0.f && !(s.softcap >= kLeastCap && s.softcap <= kLargestCap))
    return inval("softcap must be 0 (none) or from 1e-6 to 1024");
  if (misaligned(s.slopes, 4)) return inval("slopes must be 4-byte aligned");
  return GM_OK;
}

// The query rows of a call fit one launch.
bool cached_fits(int B, int Sq, int n_heads) {
  return static_cast<double>(B) * Sq * n_heads < 16777216.0;
}

// The query rows of a call over pages fit a launch.
bool paged_fits(int B, int n, int n_heads, bool packed) {
  const double tokens = packed ? static_cast<double>(n) + B : static_cast<double>(B) * n;
  return tokens * n_heads < 16777216.0;
}

int check_window(int window) {
  return window < 0 || window > kPositions ? inval("window must be 0 (none) or up to 2^24") : GM_OK;
}

int check_paged_cache(const gm_paged_cache* c) {
  if (!c) return inval("cache is NULL");
  if (int rc = check_dtype(c->dtype)) return rc;
  if (int rc = check_head_dim(c->head_dim)) return rc;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return inval("page_size must be a power of two from 16 to 256");
  if (c->pages < 1 || c->heads < 1 || c->heads > (1 << 16))
    return inval("cache pages and heads must be positive");
  if (!c->k || !c->v) return inval("a cache pointer is NULL");
  if (misaligned(c->k, 16) || misaligned(c->v, 16)) return inval("cache memory must be 16-byte aligned");
  return GM_OK;
}

// Sizes alone: what the workspace depends on.
int check_paged_sizes(const gm_paged_cache* c, int B, int n, int width) {
  if (int rc = check_paged_cache(c)) return rc;
  if (B < 0 || B > (1 << 20)) return inval("B must be at most 2^20");
  if (n < 0 || n >= kPositions) return inval("n must be below 2^24");
  if (width < 1 || static_cast<int64_t>(width) * c->page_size > kPositions)
    return inval("the table's width times page_size must be positive and at most 2^24");
  return GM_OK;
}

int check_paged_rows(const gm_paged_cache* c, const gm_paged_rows& r) {
  if (int rc = check_paged_sizes(c, r.B, r.n, r.width)) return rc;
  if (!r.offsets && static_cast<double>(r.B) * r.n >= kPositions) return inval("B * n must be below 2^24");
  if (r.B == 0 || r.n == 0) return GM_OK;
  if (!r.table || !r.lengths) return inval("table or lengths is NULL");
  if (misaligned(r.table, 4) || misaligned(r.lengths, 4) || misaligned(r.offsets, 4))
    return inval("int32 arrays must be 4-byte aligned");
  if (r.B > 1 && (r.table_stride < 0 || r.table_stride >= (int64_t(1) << 40)))
    return inval("table_stride is out of range");
  return GM_OK;
}

// The tensors of new tokens: packed ones are one sequence of n.
int check_paged_tensor(const gm_tensor& t, const gm_paged_cache* c, const gm_paged_rows& r, int heads,
                       bool output) {
  return check_tensor(t, c->dtype, r.offsets ? 1 : r.B, r.n, heads, c->head_dim, output);
}

bool same_place(const gm_tensor& x, const gm_tensor& y, const gm_paged_rows& r, int heads) {
  return x.p == y.p && (r.offsets || r.B == 1 || x.batch == y.batch) && (r.n == 1 || x.token == y.token) &&
         (heads == 1 || x.head == y.head);
}

int launched() {
  HIP_TRY(hipGetLastError());
  return GM_OK;
}

}  // namespace

extern "C" {

int gm_kv_write(const gm_kv_cache* cache, int32_t dtype, int32_t B, int32_t n, gm_tensor k,
                gm_tensor v, const int32_t* start, const int32_t* count, const int32_t* mask,
                hipStream_t stream) {
  if (int rc = check_rows(cache, dtype, B, n, k, v, start, count, mask, false)) return rc;
  if (mask && !cache->valid) return inval("a mask needs a cache with valid bytes");
  if (B == 0 || n == 0) return GM_OK;
  launch_kv_write(*cache, dtype, B, n, k, v, start, count, mask, stream);
  return launched();
}

int gm_kv_read(const gm_kv_cache* cache, int32_t dtype, int32_t B, int32_t n, const int32_t* start,
               const int32_t* count, gm_tensor k, gm_tensor v, hipStream_t stream) {
  if (int rc = check_rows(cache, dtype, B, n, k, v, start, count, nullptr, true)) return rc;
  if (B == 0 || n == 0) return GM_OK;
  if (k.p == v.p) return inval("k and v overlap");
  launch_kv_read(*cache, dtype, B, n, start, count, k, v, stream);
  return launched();
}

uint64_t gm_attention_cached_workspace(const gm_kv_cache* cache, int32_t dtype, int32_t B,
                                       int32_t Sq, int32_t n_heads) {
  if (check_cache(cache) || check_dtype(dtype) || B < 1 || B > cache->batch || Sq < 1 ||
      Sq > cache->max_seq || n_heads < 1 || n_heads % cache->heads || !cached_fits(B, Sq, n_heads))
    return 0;
  return attention_cached_workspace(*cache, dtype, B, Sq, n_heads);
}

int gm_attention_cached(const gm_cached_attention* a, hipStream_t stream) {
  if (!a) return inval("arguments are NULL");
  const gm_kv_cache* c = a->cache;
  int rc = check_cache(c);
  if (rc || (rc = check_dtype(a->dtype)) || (rc = check_scores(a->scores))) return rc;
  if (a->B < 0 || a->B > c->batch) return inval("B must be at most the cache's batch");
  if (a->Sq < 0 || a->Sq > c->max_seq) return inval("Sq must be at most the cache's max_seq");
  if (a->n_heads < 1 || a->n_heads % c->heads)
    return inval("n_heads must be a multiple of the cache's heads");
  if ((rc = check_tensor(a->q, a->dtype, a->B, a->Sq, a->n_heads, c->head_dim, false)) ||
      (rc = check_tensor(a->out, a->dtype, a->B, a->Sq, a->n_heads, c->head_dim, true)))
    return rc;
  if (a->B == 0 || a->Sq == 0) return GM_OK;
  if (!a->lengths || misaligned(a->lengths, 4)) return inval("lengths must be a 4-byte aligned pointer");
  if (!cached_fits(a->B, a->Sq, a->n_heads)) return inval("B * Sq * n_heads must be below 2^24");
  const uint64_t need = attention_cached_workspace(*c, a->dtype, a->B, a->Sq, a->n_heads);
  if (need && (!a->workspace || misaligned(a->workspace, 16) || a->workspace_bytes < need))
    return inval("workspace is NULL, misaligned or smaller than gm_attention_cached_workspace");
  if (a->out.p == a->q.p) return inval("out and q overlap");
  launch_attention_cached(*a, stream);
  return launched();
}

int gm_attention(const gm_prompt_attention* a, hipStream_t stream) {
  if (!a) return inval("arguments are NULL");
  int rc = check_dtype(a->dtype);
  if (rc || (rc = check_head_dim(a->head_dim)) || (rc = check_scores(a->scores))) return rc;
  if (a->B < 0 || a->Sq < 0 || a->Sk < 0) return inval("sizes may not be negative");
  if (a->kv_heads < 1 || a->n_heads < 1 || a->n_heads % a->kv_heads)
    return inval("n_heads must be a multiple of kv_heads");
  const int64_t off = a->q_offset;
  if (a->Sk >= kPositions || (off < 0 ? -off : off) + a->Sq >= kPositions)
    return inval("positions must be below 2^24");
  if ((rc = check_tensor(a->q, a->dtype, a->B, a->Sq, a->n_heads, a->head_dim, false)) ||
      (rc = check_tensor(a->k, a->dtype, a->B, a->Sk, a->kv_heads, a->head_dim, false)) ||
      (rc = check_tensor(a->v, a->dtype, a->B, a->Sk, a->kv_heads, a->head_dim, false)) ||
      (rc = check_tensor(a->out, a->dtype, a->B, a->Sq, a->n_heads, a->head_dim, true)))
    return rc;
  if (a->Sk > 0 && !a->q_doc != !a->k_doc) return inval("q_doc and k_doc go together");
  if (a->prefix && !a->causal) return inval("prefix needs causal");
  if (misaligned(a->key_mask, 4) || misaligned(a->q_doc, 4) || misaligned(a->k_doc, 4) ||
      misaligned(a->prefix, 4))
    return inval("int32 arrays must be 4-byte aligned");
  if (a->B == 0 || a->Sq == 0) return GM_OK;
  // a launch has fewer than 2^32 threads, 256 for 32 query rows of a head
  if (static_cast<double>(a->B) * a->n_heads * ((a->Sq + 31) / 32) >= 16777216.0)
    return inval("B * n_heads * ceil(Sq / 32) must be below 2^24");
  if (a->out.p == a->q.p || (a->Sk > 0 && (a->out.p == a->k.p || a->out.p == a->v.p)))
    return inval("out and an input overlap");
  launch_attention_prompt(*a, stream);
  return launched();
}

int gm_paged_append(const gm_paged_append_args* a, hipStream_t stream) {
  if (!a) return inval("arguments are NULL");
  const gm_paged_cache* c = a->cache;
  const gm_paged_rows& r = a->rows;
  int rc = check_paged_rows(c, r);
  if (rc || (rc = check_paged_tensor(a->k, c, r, c->heads, false)) ||
      (rc = check_paged_tensor(a->v, c, r, c->heads, false)))
    return rc;
  if (a->n_q_heads < 0 || a->n_q_heads > (1 << 16)) return inval("n_q_heads must be from 0 to 2^16");
  if (a->n_q_heads > 0 && ((rc = check_paged_tensor(a->q, c, r, a->n_q_heads, false)) ||
                           (rc = check_paged_tensor(a->q_out, c, r, a->n_q_heads, true))))
    return rc;
  if (a->rot < 0 || a->rot > c->head_dim || a->rot % 16)
    return inval("rot must be 0 or a multiple of 16 up to head_dim");
  if (r.B == 0 || r.n == 0) return GM_OK;
  if (a->rot > 0) {
    if (!a->cos || !a->sin || misaligned(a->cos, 16) || misaligned(a->sin, 16))
      return inval("cos and sin must be 16-byte aligned pointers");
    if (a->positions < static_cast<int64_t>(r.width) * c->page_size)
      return inval("cos and sin must hold every position of the table (width * page_size)");
  }
  for (const void* t : {a->k.p, a->v.p})
    if (t == c->k || t == c->v) return inval("k or v and the cache overlap");
  if (a->n_q_heads > 0) {
    const void* o = a->q_out.p;
    if (o == a->k.p || o == a->v.p || o == c->k || o == c->v) return inval("q_out and another tensor overlap");
    if (o == a->q.p && !same_place(a->q, a->q_out, r, a->n_q_heads))
      return inval("q_out may be q itself, not another view of it");
  }
  launch_paged_append(*a, stream);
  return launched();
}

uint64_t gm_paged_attention_workspace(const gm_paged_cache* cache, int32_t B, int32_t n, int32_t width,
                                      int32_t n_heads, int32_t window, int32_t packed) {
  if (check_paged_sizes(cache, B, n, width) || B < 1 || n < 1 || n_heads < 1 || n_heads % cache->heads ||
      check_window(window) || !paged_fits(B, n, n_heads, packed != 0))
    return 0;
  return paged_attention_workspace(*cache, B, n, width, n_heads, window, packed != 0);
}

int gm_paged_attention(const gm_paged_attention_args* a, hipStream_t stream) {
  if (!a) return inval("arguments are NULL");
  const gm_paged_cache* c = a->cache;
  const gm_paged_rows& r = a->rows;
  int rc = check_paged_rows(c, r);
  if (rc || (rc = check_scores(a->scores))) return rc;
  if (a->n_heads < 1 || a->n_heads % c->heads) return inval("n_heads must be a multiple of the cache's heads");
  if ((rc = check_window(a->window))) return rc;
  if ((rc = check_paged_tensor(a->q, c, r, a->n_heads, false)) ||
      (rc = check_paged_tensor(a->out, c, r, a->n_heads, true)))
    return rc;
  if (r.B == 0 || r.n == 0) return GM_OK;
  if (!paged_fits(r.B, r.n, a->n_heads, r.offsets != nullptr))
    return inval("the query rows (tokens * n_heads, and sequences * n_heads if packed) must be below 2^24");
  if (a->out.p == a->q.p || a->out.p == c->k || a->out.p == c->v) return inval("out and an input overlap");
  const uint64_t need = paged_attention_workspace(*c, r.B, r.n, r.width, a->n_heads, a->window, r.offsets != nullptr);
  if (need && (!a->workspace || misaligned(a->workspace, 16) || a->workspace_bytes < need))
    return inval("workspace is NULL, misaligned or smaller than gm_paged_attention_workspace");
  launch_paged_attention(*a, stream);
  return launched();
}

}  // extern "C"
