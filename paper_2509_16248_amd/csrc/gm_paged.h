// gm_paged.h -- what the kernels over a paged KV cache (gm.h, gm_paged_cache)
// share: a call's sequences, their division into work, places in the cache, and
// the exact walk of one query row.
#pragma once
#include <type_traits>

#include "gm_flash.h"
#include "gm_ops.h"

namespace gm {

constexpr float kPagedLog2e = 1.4426950408889634f;

// fp16 weights go into the matrix products times 2^7 (the largest is 2^15): fewer fall below the
// type's smallest normal.  Their sum is then that much too large, which a row's output, divided by
// it, does not show; a part in the workspace holds the sum without the factor (times kWeightDown),
// as paged_row returns it, so that parts computed either way may be joined.
template <typename T> constexpr float kWeightUp = std::is_same<T, f16_t>::value ? 7.f : 0.f;
template <typename T> constexpr float kWeightDown = std::is_same<T, f16_t>::value ? 0x1p-7f : 1.f;

// Memory that no kernel writes while it is read here, by a scalar load where the
// address is the same for every lane.
__device__ __forceinline__ int32_t const_load(const int32_t* p) {
  typedef const __attribute__((address_space(4))) int32_t* cptr;
  return *(cptr)reinterpret_cast<uintptr_t>(p);
}

// 16 bytes of LDS, as lds_read_tr16 reads them: the compiler makes such a read wait for every
// copy into LDS in flight, and for the read before it.  lgkm_wait16() must precede any use.
template <int OFF>
__device__ __forceinline__ u32x4 lds_read16(uint32_t addr) {
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF) : "memory");
  return v;
}
// Wait until at most N LDS reads are outstanding, then tie two values to the wait.
template <int N>
__device__ __forceinline__ void lgkm_wait16(u32x4 (&v)[2]) {
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"i"(N) : "memory");
  asm volatile("" : "+v"(v[0]), "+v"(v[1]));
}

// One sequence of an attention call: its query rows, n tokens from row row0 of the packed
// rows, its keys [lo, kend) that any of them may see, and the position p0 of the first.
struct PagedSeq {
  int row0, n, p0, kend, lo;
};
__device__ __forceinline__ PagedSeq paged_seq(const gm_paged_attention_args& a, const gm_paged_cache& c, int b) {
  PagedSeq s;
  s.row0 = 0;
  s.n = a.rows.n;
  if (a.rows.offsets) {
    const int o0 = const_load(a.rows.offsets + b), o1 = const_load(a.rows.offsets + b + 1);
    s.row0 = o0 < 0 ? 0 : o0 < a.rows.n ? o0 : a.rows.n;
    s.n = (o1 < a.rows.n ? o1 : a.rows.n) - s.row0;
    s.n = s.n > 0 ? s.n : 0;
  }
  const int len = const_load(a.rows.lengths + b), cap = a.rows.width * c.page_size;
  s.kend = len < 0 ? 0 : len < cap ? len : cap;
  // lengths may hold anything: a token that lies past the table by the window sees nothing, and
  // without a window everything, with the same weights wherever it is (a bias falls by as much for
  // every key), so positions end there and the sums made of them stay below 2^26
  const int last = cap + a.window;
  s.p0 = (len < 0 ? 0 : len) - s.n;
  s.p0 = s.p0 < last ? s.p0 : last;
  s.lo = a.window > 0 && s.p0 - a.window + 1 > 0 ? s.p0 - a.window + 1 : 0;
  s.lo = s.lo < s.kend ? s.lo : s.kend;
  return s;
}
template <typename T>
__device__ __forceinline__ T* paged_row_at(const gm_tensor& t, const gm_paged_rows& r, int b, int row0, int i, int h) {
  return static_cast<T*>(t.p) + (r.offsets ? 0 : b * t.batch) + static_cast<int64_t>(row0 + i) * t.token + h * t.head;
}

// Elements from the start of a page to the rows of one head's slot 0.
__device__ __forceinline__ int64_t paged_base(const gm_paged_cache& c, int page, int kvh) {
  return (static_cast<int64_t>(page) * c.heads + kvh) * c.page_size * c.head_dim;
}

// The sequence of packed row `row`, by one wavefront: how many end at or before it (B: none
// holds it; nor does the one found, if it begins behind it).  Appending a token of each of 64
// sequences (32/8 heads of 128) takes 4.8 us, with n each 4.6; of 512 6.8 and 5.4, of 4096 40.7 and 19.4.
__device__ __forceinline__ int paged_sequence_of(const gm_paged_rows& r, int row) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int b0 = 0; b0 < r.B; b0 += 64) {
    const int end = b0 + lane < r.B ? r.offsets[b0 + lane + 1] : row + 1;
    const int some = __builtin_popcountll(__ballot(end <= row));
    before += some;
    if (some < 64) break;
  }
  return __builtin_amdgcn_readfirstlane(before);
}

// Running sum over the lanes, each with those before it (wave_sum's steps).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, ROWS == 0xf);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += dpp_or_0<0x111, 0xf>(v);   // row_shr:1
  v += dpp_or_0<0x112, 0xf>(v);   // row_shr:2
  v += dpp_or_0<0x114, 0xf>(v);   // row_shr:4
  v += dpp_or_0<0x118, 0xf>(v);   // row_shr:8
  v += dpp_or_0<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3
  v += dpp_or_0<0x143, 0xc>(v);   // row_bcast:31 into rows 2 and 3
  return v;
}

// One query row (token i of sequence b, head h) over the keys [k0, k1) by one
// wavefront, a key per lane: two passes over the keys, the largest score and the
// weights' sum, then the output, of weights that add up to 1, so that it overflows only
// where it has to.  A hidden key is skipped, so that nothing its value holds can reach
// the sums.  store(channel, value) for every channel; the row's largest score (log2
// units) and its sum of exp2(score - largest) are returned.
template <typename T, int HD, typename F>
__device__ __forceinline__ f32x2 paged_row(const gm_paged_attention_args& a, const gm_paged_cache& c,
                                           const PagedSeq& s, int b, int h, int i, int k0, int k1, F store) {
  constexpr int CL = (HD + 63) / 64;   // channels per lane
  const int lane = threadIdx.x & 63, lg = 31 - __builtin_clz(c.page_size);
  const int kvh = h / (a.n_heads / c.heads), qpos = s.p0 + i;
  const T* q = paged_row_at<const T>(a.q, a.rows, b, s.row0, i, h);
  const int32_t* table = a.rows.table + b * a.rows.table_stride;
  const float slope = a.scores.slopes ? a.scores.slopes[h] : 0.f;
  k1 = k1 < qpos + 1 ? k1 : qpos + 1;
  k1 = k1 < s.kend ? k1 : s.kend;
  if (a.window > 0 && k0 < qpos - a.window + 1) k0 = qpos - a.window + 1;
  auto place = [&](int j) -> int64_t {   // of key j's first channel; -1: hidden
    if (j >= k1) return -1;
    const int page = table[j >> lg];
    if (page < 0 || page >= c.pages) return -1;
    return paged_base(c, page, kvh) + (j & (c.page_size - 1)) * HD;
  };
  auto score = [&](int j, int64_t at) {
    const T* k = static_cast<const T*>(c.k) + at;
    float x = 0.f;
#pragma unroll 4
    for (int e = 0; e < HD; ++e) x = fmaf(to_f32(q[e]), to_f32(k[e]), x);
    return modify_score(x * a.scores.scale, a.scores.softcap, slope, static_cast<float>(qpos - j));
  };
  float m = -INFINITY, l = 0.f;
  for (int j0 = k0; j0 < k1; j0 += 64) {
    const int64_t at = place(j0 + lane);
    if (at < 0) continue;
    const float x = score(j0 + lane, at);
    if (x == -INFINITY) continue;
    const float mn = fmaxf(m, x);
    l = (m == -INFINITY ? l : l * expf(m - mn)) + expf(x - mn);   // (a NaN stays)
    m = mn;
  }
  const float M = wave_max(m);
  l = wave_sum(m == -INFINITY ? l : l * expf(m - M));
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float o[CL] = {};
  for (int j0 = k0; j0 < k1; j0 += 64) {
    const int64_t at = place(j0 + lane);
    float p = 0.f;
    if (at >= 0) {
      const float x = score(j0 + lane, at);
      p = x == -INFINITY ? 0.f : expf(x - M) * inv;
    }
    for (int t = 0; t < 64 && j0 + t < k1; ++t) {
      const float pt = __shfl(p, t, 64);
      const int64_t vt = __shfl(at, t, 64);
      if (vt < 0) continue;
      const T* v = static_cast<const T*>(c.v) + vt;
#pragma unroll
      for (int e = 0; e < CL; ++e)
        if (lane + 64 * e < HD) o[e] = fmaf(pt, to_f32(v[lane + 64 * e]), o[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < CL; ++e)
    if (lane + 64 * e < HD) store(lane + 64 * e, l == 0.f ? 0.f : o[e]);
  return f32x2{M * kPagedLog2e, l};
}

// f(head size, storage type) as compile-time values.
template <typename F>
void by_paged_cache(const gm_paged_cache& c, F f) {
  auto head = [&](auto t) {
    if (c.head_dim == 32) f(t, std::integral_constant<int, 32>());
    else if (c.head_dim == 64) f(t, std::integral_constant<int, 64>());
    else f(t, std::integral_constant<int, 128>());
  };
  if (c.dtype == kF32) head(float());
  else if (c.dtype == kBF16) head(bf16_t());
  else head(f16_t());
}

// gm_paged_prompt.hip: 16-bit chunks of many rows.  Sequences of at most `few` query rows
// per key head are left to the rows kernel (0: none are).
void launch_paged_prompt(const gm_paged_attention_args& a, int few, hipStream_t s);
uint64_t paged_prompt_workspace(const gm_paged_cache& c, int B, int n, int width, int n_heads, int few, bool packed);

}  // namespace gm
