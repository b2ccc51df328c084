// gm_paged.hip -- a KV cache in pages (gm.h, gm_paged_cache): new rows stored with
// their rotation applied on the way, and attention of a few new tokens over it.
// Chunks of many tokens in 16 bits: gm_paged_prompt.hip.
#include <math.h>

#include <algorithm>

#include "gm_device.h"
#include "gm_paged.h"

namespace gm {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ append
//
// Moves bytes: a token's query, key and value rows once each way, and its row of cosines and
// sines.  What a small call waits for is the chain offsets - length - table entry - store, so
// the rows are fetched before their place is looked up (8 tokens of 12 heads of 64: 3.8 ->
// 3.4 us; eight packed chunks, 16,000 tokens of 32/8 heads of 128, fp16, 86 -> 78 us, 5.2 TB/s;
// 2048 tokens of 32 heads 17.8 us, 5.7 TB/s, partly from the Infinity Cache).
// TPT threads, a wavefront or the workgroup, take one token: its query, key and value heads in
// one line, a thread 16 channels of a head, the two halves of 8 pairs (lo, hi) that turn
// together (of channels that do not turn: 16 in a row).  TPT is a multiple of a head's
// threads, so a thread's channels and its cosines and sines are the same for all of its heads.
template <typename T> struct Half8 {       // 8 channels
  static constexpr int NV = static_cast<int>(sizeof(T)) / 2;
  u32x4 raw[NV];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = reinterpret_cast<const u32x4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) reinterpret_cast<u32x4*>(p)[i] = raw[i];
  }
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(raw)[i]); }
  __device__ __forceinline__ void set(int i, float x) { reinterpret_cast<T*>(raw)[i] = from_f32<T>(x); }
};

template <typename T, int HD, int TPT>
__global__ __launch_bounds__(256) void k_paged_append(gm_paged_append_args a, gm_paged_cache c, int tokens) {
  constexpr int LPR = HD / 16, U = 4, STEP = TPT / LPR;
  const gm_paged_rows& r = a.rows;
  const int nq = a.n_q_heads, heads = nq + 2 * c.heads;
  const int row = TPT == 256 ? blockIdx.x : blockIdx.x * (256 / TPT) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPT);
  if (row >= tokens) return;
  const int ch = threadIdx.x % LPR;
  const bool turns = ch < a.rot / 16;
  // packed rows are one sequence as far as their tensors go
  const int first = r.offsets ? 0 : row / r.n, i = r.offsets ? row : row - first * r.n;
  Half8<T> lo[U], hi[U];
  // of pairs that turn, and of 16 channels in a row (values: from the head's start)
  auto from = [&](int h) { return turns && h < nq + c.heads ? 8 * ch : 16 * ch; };
  auto to = [&](int h) { return turns && h < nq + c.heads ? 8 * ch + a.rot / 2 : 16 * ch + 8; };
  auto fetch = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * STEP;
      if (h >= heads) break;
      const gm_tensor& t = h < nq ? a.q : h < nq + c.heads ? a.k : a.v;
      const int hh = h < nq ? h : h < nq + c.heads ? h - nq : h - nq - c.heads;
      const T* x = static_cast<const T*>(t.p) + first * t.batch + i * t.token + hh * t.head;
      lo[u].load(x + from(h));
      hi[u].load(x + to(h));
    }
  };
  const int h1 = threadIdx.x % TPT / LPR;
  fetch(h1);                                 // (on their way while the place is looked up)
  // ---- whose token this is, and its position
  const int b = r.offsets ? paged_sequence_of(r, row) : first;
  if (b >= r.B) return;
  int end = r.n, before = i;                 // of the sequence's rows, and the token's place in them
  if (r.offsets) {
    const int o1 = const_load(r.offsets + b + 1);
    if (row < const_load(r.offsets + b)) return;
    end = o1 < r.n ? o1 : r.n;
  }
  const int64_t pos = static_cast<int64_t>(const_load(r.lengths + b)) - end + before;
  const bool inside = pos >= 0 && pos < static_cast<int64_t>(r.width) * c.page_size;
  const int p = inside ? static_cast<int>(pos) : 0, lg = 31 - __builtin_clz(c.page_size);
  float cosv[8], sinv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cosv[j] = 1.f;
    sinv[j] = 0.f;
  }
  if (turns && inside) {
    const int64_t at = static_cast<int64_t>(p) * (a.rot / 2) + 8 * ch;
    Half8<float> x;
    x.load(a.cos + at);
#pragma unroll
    for (int j = 0; j < 8; ++j) cosv[j] = x.get(j);
    x.load(a.sin + at);
#pragma unroll
    for (int j = 0; j < 8; ++j) sinv[j] = x.get(j);
  }
  const int page = const_load(r.table + b * r.table_stride + (p >> lg));
  const bool stored = inside && page >= 0 && page < c.pages;
  const int64_t slot = paged_base(c, stored ? page : 0, 0) + (p & (c.page_size - 1)) * HD;
  const int64_t head_step = static_cast<int64_t>(c.page_size) * HD;
  for (int h0 = h1; h0 < heads; h0 += U * STEP) {
    if (h0 != h1) fetch(h0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * STEP;
      if (h >= heads) break;
      if (turns && h < nq + c.heads) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = lo[u].get(j), y = hi[u].get(j);
          lo[u].set(j, fmaf(x, cosv[j], -(y * sinv[j])));
          hi[u].set(j, fmaf(y, cosv[j], x * sinv[j]));
        }
      }
      T* out;
      if (h < nq) {
        if (!inside) {
#pragma unroll
          for (int e = 0; e < Half8<T>::NV; ++e) lo[u].raw[e] = hi[u].raw[e] = u32x4{0, 0, 0, 0};
        }
        out = static_cast<T*>(a.q_out.p) + first * a.q_out.batch + i * a.q_out.token + h * a.q_out.head;
      } else {
        if (!stored) continue;
        const bool key = h < nq + c.heads;
        out = static_cast<T*>(key ? c.k : c.v) + slot + (h - nq - (key ? 0 : c.heads)) * head_step;
      }
      lo[u].store(out + from(h));
      hi[u].store(out + to(h));
    }
  }
}

// ------------------------------------------------------------ attention of a few tokens
//
// Reads every seen key and value once per block of rows: memory bounds it, at 5.3 to 5.5 TB/s
// of the long caches (a large copy moves 4.89).  The rows of a key head (its query heads times
// the new tokens) come in blocks of R = 16 or 32; an item is such a block.  Its keys go through in tiles; where items are few they are
// cut up: all tiles of all items in one line, and each of `wgs` workgroups takes an equal
// part of it, whatever the lengths are (one of 32 sequences long, the others short).  A
// workgroup then has the end of one item, whole ones, and the start of another; the two
// cut ones leave, per query row, the largest score m (log2 units), the sum l of its
// exp2(score - m) and their own normalised output o in the workspace, and k_paged_join adds
// sum(w o) / sum(w), w = l exp2(m - largest m), in order of the keys.
struct PagedPlan {
  int G;         // query heads of a key head
  int blocks;    // row blocks of a key head; 0: packed, each sequence has its own
  int few;       // sequences of more rows than this are another kernel's (0: none are)
  int wgs;       // workgroups that share all tiles; 0: a workgroup an item
  int items;     // items there are at the most
  int joined;    // rows of a block at the most
};

constexpr int kMostParts = 64;     // workgroups that share an item

template <int R, int UNIT>
__device__ __forceinline__ void paged_weight(const gm_paged_attention_args& a, const gm_paged_cache& c,
                                             const PagedPlan& p, const PagedSeq& s, int& blocks, int& tiles) {
  const int rows = s.n * p.G;
  blocks = p.few && rows > p.few ? 0 : (rows + R - 1) / R;
  // (a sequence without keys still has rows to clear)
  tiles = (s.kend - (s.lo & ~31) + UNIT - 1) / UNIT;
  tiles = tiles > 0 ? tiles : 1;
}

// Tiles a workgroup takes of all, where an item has at most `most`.
__device__ __forceinline__ int paged_share(const PagedPlan& p, unsigned all, unsigned most) {
  const unsigned even = (all + p.wgs - 1) / p.wgs, least = (most + kMostParts - 3) / (kMostParts - 2);
  return __builtin_amdgcn_readfirstlane(even > least ? even : least);
}

// Where in the line of all sequences' items and tiles something lies.
struct PagedFound {
  int b;                       // its sequence; -1: none
  unsigned items, tiles;       // those of the sequences before
  unsigned all_tiles;
  unsigned at;                 // the item, or the tile
  int per;                     // tiles a workgroup takes
};
// By one wavefront: the sequence that item x (FIND_ITEM), or workgroup x's first or last
// tile falls into.
enum { FIND_ITEM, FIND_FIRST, FIND_LAST };
template <int R, int UNIT, int WHAT>
__device__ __forceinline__ PagedFound paged_find(const gm_paged_attention_args& a, const gm_paged_cache& c,
                                                 const PagedPlan& p, unsigned x) {
  constexpr bool by_tile = WHAT != FIND_ITEM;
  const int lane = threadIdx.x & 63, each = (a.rows.B + 63) / 64;
  unsigned items = 0, tiles = 0, most = 0;
  for (int e = 0; e < each; ++e) {
    const int b = lane * each + e;
    if (b >= a.rows.B) break;
    int nb, nt;
    paged_weight<R, UNIT>(a, c, p, paged_seq(a, c, b), nb, nt);
    items += static_cast<unsigned>(nb) * c.heads;
    tiles += static_cast<unsigned>(nb) * c.heads * nt;
    most = nb && static_cast<unsigned>(nt) > most ? nt : most;
  }
  const unsigned si = wave_scan(items), st = wave_scan(tiles);
  PagedFound f;
  f.all_tiles = __builtin_amdgcn_readlane(st, 63);
  f.per = p.wgs ? paged_share(p, f.all_tiles, wave_max_u32(most)) : 0;
  unsigned at = by_tile ? x * f.per : x;
  if (WHAT == FIND_LAST && at < f.all_tiles) at = (at + f.per < f.all_tiles ? at + f.per : f.all_tiles) - 1;
  f.at = at;
  const unsigned mine = by_tile ? tiles : items, end = by_tile ? st : si;
  const unsigned long long hit = __ballot(at < end && at >= end - mine);
  f.b = -1;
  if (hit == 0) return f;
  const int l = __builtin_ctzll(hit);
  f.items = __builtin_amdgcn_readlane(si - items, l);
  f.tiles = __builtin_amdgcn_readlane(st - tiles, l);
  for (int b = l * each; b < a.rows.B; ++b) {  // (the lane's sequences hold it)
    int nb, nt;
    paged_weight<R, UNIT>(a, c, p, paged_seq(a, c, b), nb, nt);
    const unsigned i = static_cast<unsigned>(nb) * c.heads, t = i * nt;
    if (at < (by_tile ? f.tiles + t : f.items + i)) {
      f.b = __builtin_amdgcn_readfirstlane(b);
      return f;
    }
    f.items += i;
    f.tiles += t;
  }
  return f;
}

// (m, l, o[HD]) of a row of a workgroup's cut item: slot 0 that begins before it, 1 after.
template <int R, int HD>
__device__ __forceinline__ float* paged_part(const gm_paged_attention_args& a, unsigned wg, int slot, int row) {
  return static_cast<float*>(a.workspace) + ((static_cast<size_t>(wg) * 2 + slot) * R + row) * (HD + 2);
}

// Products of 16 x 16 with the type's k, fp32 sums: A and B of a lane (n = lane % 16, g =
// lane / 16), 16 bytes of each.
template <typename T> struct Mfma16;
template <> struct Mfma16<bf16_t> {
  static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mfma16<f16_t> {
  static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mfma16<float> {
  static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
};

// BYTES bytes (4, 8, 16 or 32) as 32-bit words.
template <int BYTES>
__device__ __forceinline__ void load_row(const char* p, uint32_t* w) {
  if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (BYTES == 8) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    w[0] = v[0];
    w[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
    }
  }
}

constexpr int rows_waves(int hd, int nset) { return hd == 128 || nset == 2 ? 2 : hd == 64 ? 3 : 4; }

// S[key][row] = K Q^T and O^T[channel][row] += V^T P^T on products of 16 x 16, a wavefront
// taking every NWV-th tile of KB keys, without LDS or barrier before the end.
// Keys 16 u + m of a tile are row m of product u: a load's keys lie in one page
// (pages are multiples of 16), so that its address is a scalar and a lane's fixed offset.
// A lane (n, g) ends with the scores of keys 16 u + 4 g + r of row n, and those are the k
// slots of its operand of P: P needs no exchange.  V comes in rows, HD / 16 channels of a
// key a lane, row m of product e being channel (HD / 16) m + e; in 16 bits a byte permute per
// word puts two keys of a channel together.
// 16-bit weights are rounded to the type for the second product (half a step of each, up to 2^-8
// or 2^-11 of it; their sum takes them unrounded): its operands are 16-bit.
// The two tiles of NSET = 1 take 64 registers each at 128 channels; with 32 rows there is one,
// whose K and V are fetched again as soon as each has been used.
// The maximum m moves lazily (by more than 2^8).  Hidden keys have weight 0, and values that
// no row sees are cleared (a page's unused end may hold anything); rows that still come out
// not finite are computed again by paged_row, which skips what is hidden.
template <typename T, int HD, int NSET, bool CAP, int NWV>
__global__ __launch_bounds__(64 * NWV) __attribute__((amdgpu_waves_per_eu(rows_waves(HD, NSET), rows_waves(HD, NSET))))
void k_paged_rows(gm_paged_attention_args a, gm_paged_cache c, PagedPlan plan) {
  constexpr int ES = sizeof(T), NU = ES == 4 ? 1 : 2, KB = 16 * NU, NS = 4 * NU;
  constexpr int R = 16 * NSET, UNIT = NWV * KB;
  constexpr int KC = HD * ES / 64;                  // 16-byte chunks of a lane's K row
  constexpr int VB = HD / 16 * ES, VW = VB / 4;     // bytes, words of its V rows
  constexpr int NI = HD / 16;                       // products of O
  constexpr int RB = HD * ES;                       // bytes of a row
  constexpr bool F32 = ES == 4;
  constexpr int SO = HD + 4;                        // floats of a row of s_o
  __shared__ __attribute__((aligned(16))) float s_o[NWV][R][SO];
  __shared__ __attribute__((aligned(16))) float s_f[NSET == 2 ? R : 1][NWV];
  __shared__ float s_m[NWV][R], s_l[NWV][R], s_M[NSET == 2 ? R : 1], s_L[NSET == 2 ? R : 1];
  __shared__ uint32_t s_odd;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int lg = 31 - __builtin_clz(c.page_size);
  const int64_t page_bytes = static_cast<int64_t>(c.heads) * c.page_size * RB;
  const float c2 = CAP ? (F32 ? a.scores.scale / a.scores.softcap : a.scores.scale * (2.f * kPagedLog2e) / a.scores.softcap)
                       : a.scores.scale * kPagedLog2e;
  const float capc = a.scores.softcap * kPagedLog2e;
  const uint32_t koff = n * RB + 16 * g, voff = 4 * g * RB + VB * n;

  // ---- rows [blk * R, ...) of key head kvh over the keys [k0, k1); part: where a cut
  // item's rows go
  auto work = [&](int b, const PagedSeq& s, int kvh, int blk, int k0, int k1, float* part) {
    const int32_t* table = a.rows.table + b * a.rows.table_stride;
    const int last_page = a.rows.width - 1;
    auto page_of = [&](int key) {
      const int at = key >> lg;
      return const_load(table + (at < last_page ? at : last_page));
    };
    struct Ids { int id[NU]; };
    auto ids_of = [&](int kb) {
      Ids x;
#pragma unroll
      for (int u = 0; u < NU; ++u) x.id[u] = page_of(kb + 16 * u);
      return x;
    };
    auto there = [&](int id) { return static_cast<unsigned>(id) < static_cast<unsigned>(c.pages); };
    auto base_of = [&](const Ids& x, int u, int kb) {
      return (there(x.id[u]) ? x.id[u] : 0) * page_bytes + (kvh * c.page_size + ((kb + 16 * u) & (c.page_size - 1))) * static_cast<int64_t>(RB);
    };
    struct Tile { u32x4 k[NU][KC]; uint32_t v[NS][VW]; };
    auto fetch_k = [&](int kb, const Ids& x, Tile& t) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const char* base = static_cast<const char*>(c.k) + base_of(x, u, kb);
#pragma unroll
        for (int e = 0; e < KC; ++e) t.k[u][e] = *reinterpret_cast<const u32x4*>(base + koff + 64 * e);
      }
    };
    auto fetch_v = [&](int kb, const Ids& x, Tile& t) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const char* base = static_cast<const char*>(c.v) + base_of(x, u, kb);
#pragma unroll
        for (int r = 0; r < 4; ++r) load_row<VB>(base + voff + r * RB, t.v[4 * u + r]);
      }
    };
    // (of the first tile, if the keys begin at 0: looked up together with the length)
    const bool known = plan.wgs == 0 && a.window == 0;
    Ids i0;
    if (known) i0 = ids_of(KB * wave);
    const int rows = s.n * plan.G, r0 = blk * R;
    const int rlast = r0 + R < rows ? r0 + R - 1 : rows - 1;
    const int qmin = s.p0 + r0 / plan.G, qmax = s.p0 + rlast / plan.G;
    k1 = k1 < qmax + 1 ? k1 : qmax + 1;
    k1 = k1 < s.kend ? k1 : s.kend;
    if (a.window > 0 && k0 < qmin - a.window + 1) k0 = (qmin - a.window + 1) & ~(KB - 1);
    int qpos[NSET], qlow[NSET];
    float slope2[NSET];
    u32x4 qf[NSET][KC];
#pragma unroll
    for (int x = 0; x < NSET; ++x) {
      const int r = r0 + 16 * x + n <= rlast ? r0 + 16 * x + n : r0;   // (columns past the last repeat the first)
      const int i = r / plan.G, h = kvh * plan.G + r - i * plan.G;
      qpos[x] = s.p0 + i;
      qlow[x] = a.window > 0 ? qpos[x] - a.window : -1;
      slope2[x] = a.scores.slopes ? a.scores.slopes[h] * kPagedLog2e : 0.f;
      const char* q = reinterpret_cast<const char*>(paged_row_at<const T>(a.q, a.rows, b, s.row0, i, h)) + 16 * g;
#pragma unroll
      for (int e = 0; e < KC; ++e) qf[x][e] = *reinterpret_cast<const u32x4*>(q + 64 * e);
    }
    float m[NSET], l[NSET];
    f32x4 o[NSET][NI];
#pragma unroll
    for (int x = 0; x < NSET; ++x) {
      m[x] = -INFINITY;
      l[x] = 0.f;
#pragma unroll
      for (int e = 0; e < NI; ++e) o[x][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // scores of the tile at kb, in log2 units
    auto scores = [&](int kb, const Tile& t, float (&sc)[NSET][NS]) {
#pragma unroll
      for (int x = 0; x < NSET; ++x)
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < KC; ++e) acc = Mfma16<T>::run(t.k[u][e], qf[x][e], acc);
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[x][4 * u + r] = acc[r];
        }
#pragma unroll
      for (int x = 0; x < NSET; ++x) {
        const float dist = static_cast<float>(qpos[x] - kb - 4 * g);
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          float y = sc[x][j] * c2;
          if constexpr (CAP) {
            if constexpr (F32) y = capc * tanhf(y);
            else y = fmaf(-2.f * capc, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y) + 1.f), capc);
          }
          sc[x][j] = fmaf(-slope2[x], dist - static_cast<float>(16 * (j / 4) + j % 4), y);
        }
      }
    };
    // masks, weights, and O += V w
    auto values = [&](int kb, const Ids& ids, Tile& t, float (&sc)[NSET][NS]) {
      bool holes = false;
#pragma unroll
      for (int u = 0; u < NU; ++u) holes = holes || !there(ids.id[u]);
      if (kb + KB - 1 > qmin || kb + KB > k1 || (a.window > 0 && kb <= qmax - a.window) || holes) {
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          const int key = kb + 16 * (j / 4) + 4 * g + j % 4;
          const bool ok = key < k1 && there(ids.id[j / 4]);
#pragma unroll
          for (int x = 0; x < NSET; ++x) sc[x][j] = ok && key <= qpos[x] && key > qlow[x] ? sc[x][j] : -INFINITY;
#pragma unroll
          for (int e = 0; e < VW; ++e) t.v[j][e] = ok ? t.v[j][e] : 0u;
        }
      }
      u32x4 pf[NSET];
#pragma unroll
      for (int x = 0; x < NSET; ++x) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < NS; ++j) top = fmaxf(top, sc[x][j]);
        if (__ballot(top > m[x] + kTau)) {
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float mn = fmaxf(m[x], top);
          const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - mn);
          l[x] *= f;
          m[x] = mn;
#pragma unroll
          for (int e = 0; e < NI; ++e) o[x][e] *= f;
        }
        const float msub = m[x] == -INFINITY ? 0.f : m[x] - kWeightUp<T>;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          sc[x][j] = __builtin_amdgcn_exp2f(sc[x][j] - msub);
          l[x] += sc[x][j];
        }
        if constexpr (!F32) {
#pragma unroll
          for (int j = 0; j < 4; ++j) pf[x][j] = pack2<T>(sc[x][2 * j], sc[x][2 * j + 1]);
        }
      }
#pragma unroll
      for (int e = 0; e < NI; ++e) {
        if constexpr (F32) {
#pragma unroll
          for (int x = 0; x < NSET; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              o[x][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(t.v[r][e]), sc[x][r], o[x][e], 0, 0, 0);
        } else {
          u32x4 f;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            f[j] = __builtin_amdgcn_perm(t.v[2 * j + 1][e / 2], t.v[2 * j][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int x = 0; x < NSET; ++x) o[x][e] = Mfma16<T>::run(f, pf[x], o[x][e]);
        }
      }
    };
    float sc[NSET][NS];
    int kb = k0 + KB * wave;
    if (!known) i0 = ids_of(kb);
    Tile t0;
    if (kb < k1) {
      fetch_k(kb, i0, t0);
      fetch_v(kb, i0, t0);
    }
    if constexpr (NSET == 1) {
      // two tiles in turn, one being worked on while the other arrives
      Tile t1;
      Ids i1 = ids_of(kb + UNIT);
      while (kb < k1) {
        if (kb + UNIT < k1) {
          fetch_k(kb + UNIT, i1, t1);
          fetch_v(kb + UNIT, i1, t1);
        }
        const Ids i2 = ids_of(kb + 2 * UNIT);
        scores(kb, t0, sc);
        values(kb, i0, t0, sc);
        kb += UNIT;
        if (kb >= k1) break;
        if (kb + UNIT < k1) {
          fetch_k(kb + UNIT, i2, t0);
          fetch_v(kb + UNIT, i2, t0);
        }
        const Ids i3 = ids_of(kb + 2 * UNIT);
        scores(kb, t1, sc);
        values(kb, i1, t1, sc);
        kb += UNIT;
        i0 = i2;
        i1 = i3;
      }
    } else {
      // one tile, its parts loaded anew as soon as they have been used
      Ids i1 = ids_of(kb + UNIT);
      for (; kb < k1; kb += UNIT) {
        const Ids i2 = ids_of(kb + 2 * UNIT);
        scores(kb, t0, sc);
        if (kb + UNIT < k1) fetch_k(kb + UNIT, i1, t0);
        values(kb, i0, t0, sc);
        if (kb + UNIT < k1) fetch_v(kb + UNIT, i1, t0);
        i0 = i1;
        i1 = i2;
      }
    }
    // ---- the wavefront's normalised output: rows 4 g + e of product x are channels
    // NI (4 g + e) + x
#pragma unroll
    for (int x = 0; x < NSET; ++x) {
      l[x] += __shfl_xor(l[x], 16, 64);
      l[x] += __shfl_xor(l[x], 32, 64);
      if (r0 + 16 * x + n > rlast) continue;
      const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v[NI];
#pragma unroll
        for (int y = 0; y < NI; ++y) v[y] = l[x] == 0.f ? 0.f : o[x][y][e] * inv;
        float* to = &s_o[wave][16 * x + n][NI * (4 * g + e)];
        if constexpr (NI == 2) *reinterpret_cast<f32x2*>(to) = f32x2{v[0], v[1]};
        else {
#pragma unroll
          for (int y = 0; y < NI; y += 4) *reinterpret_cast<f32x4*>(to + y) = f32x4{v[y], v[y + 1], v[y + 2], v[y + 3]};
        }
      }
      if (g == 0) {
        s_m[wave][16 * x + n] = m[x];
        s_l[wave][16 * x + n] = l[x];
      }
    }
    if (threadIdx.x == 0) s_odd = 0;
    __syncthreads();
    // ---- the wavefronts' sums, four channels a thread.  Their weights (over the row's sum, before
    // the products, which might pass fp32) are computed by each thread for itself where it has
    // one or two turns, and once a row, behind a barrier more, where it has up to eight.
    auto weights = [&](int row, float (&f)[NWV], float& M, float& L) {
      M = -INFINITY;
      L = 0.f;
#pragma unroll
      for (int w = 0; w < NWV; ++w) M = fmaxf(M, s_m[w][row]);
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        f[w] = s_l[w][row] == 0.f ? 0.f : s_l[w][row] * __builtin_amdgcn_exp2f(s_m[w][row] - M);
        L += f[w];
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int w = 0; w < NWV; ++w) f[w] *= inv;
    };
    if constexpr (NSET == 2) {
      if (threadIdx.x < R && r0 + static_cast<int>(threadIdx.x) <= rlast) {
        float f[NWV], M, L;
        weights(threadIdx.x, f, M, L);
#pragma unroll
        for (int w = 0; w < NWV; ++w) s_f[threadIdx.x][w] = f[w];
        s_M[threadIdx.x] = M;
        s_L[threadIdx.x] = L;
      }
      __syncthreads();
    }
    for (int e = threadIdx.x; e < R * HD / 4; e += 64 * NWV) {
      const int ch = e % (HD / 4) * 4, row = e / (HD / 4), r = r0 + row;
      if (r > rlast) break;
      float f[NWV], M, L;
      if constexpr (NSET == 2) {
#pragma unroll
        for (int w = 0; w < NWV; ++w) f[w] = s_f[row][w];
        M = s_M[row];
        L = s_L[row];
      } else {
        weights(row, f, M, L);
      }
      f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(&s_o[w][row][ch]);
        if (f[w] != 0.f) O += f[w] * v;
      }
      float odd = 0.f * L;
#pragma unroll
      for (int j = 0; j < 4; ++j) odd = fmaf(O[j], 0.f, odd);
      if (odd != 0.f) atomicOr(&s_odd, 1u << row);  // (NaN != 0)
      if (part) {
        float* to = part + row * (HD + 2) + 2 + ch;
        *reinterpret_cast<f32x2*>(to) = f32x2{O[0], O[1]};
        *reinterpret_cast<f32x2*>(to + 2) = f32x2{O[2], O[3]};
        if (ch == 0) *reinterpret_cast<f32x2*>(to - 2) = f32x2{M, L * kWeightDown<T>};
      } else {
        const int i = r / plan.G;
        T* to = paged_row_at<T>(a.out, a.rows, b, s.row0, i, kvh * plan.G + r - i * plan.G) + ch;
        if constexpr (F32) *reinterpret_cast<f32x4*>(to) = O;
        else *reinterpret_cast<u32x2*>(to) = u32x2{pack2<T>(O[0], O[1]), pack2<T>(O[2], O[3])};
      }
    }
    __syncthreads();
    const uint32_t odd = s_odd;
    if (__builtin_expect(odd != 0, 0))
      for (int row = wave; row < R; row += NWV) {
        if (!(odd >> row & 1)) continue;
        const int i = (r0 + row) / plan.G, h = kvh * plan.G + r0 + row - i * plan.G;
        T* out = paged_row_at<T>(a.out, a.rows, b, s.row0, i, h);
        const f32x2 ml = paged_row<T, HD>(a, c, s, b, h, i, k0, k1, [&](int ch, float v) {
          if (part) part[row * (HD + 2) + 2 + ch] = v;
          else out[ch] = from_f32<T>(v);
        });
        if (part && lane == 0) {
          part[row * (HD + 2)] = ml[0];
          part[row * (HD + 2) + 1] = ml[1];
        }
      }
  };

  if (plan.wgs == 0) {
    int b, kvh, blk;
    if (plan.blocks) {
      // (heads fastest: the row blocks of a head come to one XCD where the heads are a multiple
      // of 8; later tokens, which see more keys, first)
      const int heads = a.rows.B * c.heads, x = blockIdx.x / heads, y = blockIdx.x - x * heads;
      blk = plan.blocks - 1 - x;
      b = y / c.heads;
      kvh = y - b * c.heads;
    } else if (plan.few) {
      // (sequences of more rows are not ours, and others have one block)
      b = blockIdx.x / c.heads;
      kvh = blockIdx.x - b * c.heads;
      blk = 0;
      const int rows = paged_seq(a, c, b).n * plan.G;
      if (rows == 0 || rows > plan.few) return;
    } else {
      const PagedFound f = paged_find<R, UNIT, FIND_ITEM>(a, c, plan, blockIdx.x);
      if (f.b < 0) return;
      const int x = blockIdx.x - f.items;
      b = f.b;
      blk = x / c.heads;
      kvh = x - blk * c.heads;
    }
    const PagedSeq s = paged_seq(a, c, b);
    work(b, s, kvh, blk, s.lo & ~31, s.kend, nullptr);
    return;
  }
  const PagedFound f = paged_find<R, UNIT, FIND_FIRST>(a, c, plan, blockIdx.x);
  if (f.b < 0) return;
  unsigned at = blockIdx.x * static_cast<unsigned>(f.per);
  const unsigned end = at + f.per < f.all_tiles ? at + f.per : f.all_tiles;
  unsigned first = f.tiles;                     // the sequence's first tile
  for (int b = f.b; at < end && b < a.rows.B; ++b) {
    const PagedSeq s = paged_seq(a, c, b);
    int nb, nt;
    paged_weight<R, UNIT>(a, c, plan, s, nb, nt);
    const unsigned all = static_cast<unsigned>(nb) * c.heads * nt;
    while (at < end && at < first + all) {
      const int item = (at - first) / nt, t = at - first - item * nt;
      const int stop = nt - t < static_cast<int>(end - at) ? nt : t + static_cast<int>(end - at);
      const int kvh = item / nb, blk = item - kvh * nb, org = s.lo & ~31;
      float* part = t > 0 ? paged_part<R, HD>(a, blockIdx.x, 0, 0)
                          : stop < nt ? paged_part<R, HD>(a, blockIdx.x, 1, 0) : nullptr;
      work(b, s, kvh, blk, org + t * UNIT, org + stop * UNIT, part);
      __syncthreads();                          // (LDS is used again)
      at += stop - t;
    }
    first += all;
  }
}

// The parts of cut items joined.  A workgroup whose part of the line ends within an item that
// began in it is the first of that item's; here (blockIdx.x) it stands for the item, whose
// rows go to a wavefront each: the weights by a lane per part, then the parts in order.
template <typename T, int HD, int R, int UNIT>
__global__ __launch_bounds__(256) void k_paged_join(gm_paged_attention_args a, gm_paged_cache c, PagedPlan plan) {
  constexpr int CL = (HD + 63) / 64, U = 8;    // channels of a lane, parts loaded together
  const PagedFound f = paged_find<R, UNIT, FIND_LAST>(a, c, plan, blockIdx.x);
  if (f.b < 0) return;
  const PagedSeq s = paged_seq(a, c, f.b);
  int nb, nt;
  paged_weight<R, UNIT>(a, c, plan, s, nb, nt);
  const int item = (f.at - f.tiles) / nt, kvh = item / nb, blk = item - kvh * nb;
  const unsigned t0 = f.tiles + static_cast<unsigned>(item) * nt;
  const int parts = (t0 + nt - 1) / f.per - blockIdx.x + 1;       // at most kMostParts
  const int row = blockIdx.y * 4 + (threadIdx.x >> 6), r = blk * R + row, lane = threadIdx.x & 63;
  if (t0 < blockIdx.x * static_cast<unsigned>(f.per) || parts < 2 || row >= R || r >= s.n * plan.G) return;
  auto part = [&](int p) { return paged_part<R, HD>(a, blockIdx.x + p, p == 0, row); };
  float v[U][CL];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < CL; ++e)
        v[u][e] = p0 + u < parts && lane + 64 * e < HD ? part(p0 + u)[2 + lane + 64 * e] : 0.f;
  };
  fetch(0);
  const bool on = lane < parts;
  const float m = on ? part(lane)[0] : -INFINITY, l = on ? part(lane)[1] : 0.f;
  const float M = wave_max(m);
  float w = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - M);
  const float W = wave_sum(w);
  w = w == 0.f ? 0.f : w / W;
  float o[CL] = {};
  for (int p0 = 0; p0 < parts; p0 += U) {
    if (p0) fetch(p0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float wp = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), p0 + u));
#pragma unroll
      for (int e = 0; e < CL; ++e) o[e] += wp == 0.f ? 0.f : wp * v[u][e];
    }
  }
  const int i = r / plan.G;
  T* out = paged_row_at<T>(a.out, a.rows, f.b, s.row0, i, kvh * plan.G + r - i * plan.G);
#pragma unroll
  for (int e = 0; e < CL; ++e)
    if (lane + 64 * e < HD) out[lane + 64 * e] = from_f32<T>(o[e]);
}

// How a call is done.
struct PagedWay {
  PagedPlan rows;
  int nset, waves;
  bool few, many;      // the rows kernel runs, the prompt kernel does
  uint64_t rows_bytes; // workspace of the former
};

// Query rows of a key head up to which the rows kernel takes 16 bits (prompt kernel / rows
// kernel, bf16: 4 sequences of 600 and 6000 keys, 32/8 heads of 128, 36 rows 17.5 / 18.7 and
// 33.0 / 47.5; 8 of 140 and 2000, 12 heads of 64, 33 rows 7.8 / 10.7 and 26.5 / 22.2; 16 of 2000,
// 32/8 heads of 128, 64 rows 44.3 / 39.7, 132 rows 51.2 / 80.0).
constexpr int kFewRows = 32;

// Whole items, or all tiles shared out.  A CU draws 46 GB/s at the most (one item of 4000 keys,
// 8 key heads of 128, whole 44.4 us), the chip 5 TB/s; sharing costs the join's launch and the
// ends of cut items, 5 us and more (us whole / shared by 256 workgroups of 8 wavefronts / by 512
// of 4: 8 sequences of 640 keys, 12 heads of 64, 9.0 / 13.1 / 13.0; 24 of 1028, 32/8 heads of
// 128, five tokens, 24.3 / 39.6 / 43.3; 32 of 1000 25.1 / 32.0 / 33.1, of 8190 159 / 162 / 164;
// one of 1000 15.4 / 13.6 / 12.4, of 32000 with 32 key heads 350 / 98.5 / 100; four of 1500 20.6
// / 14.8 / 15.7; one of 8190 among 31 of 300 102 / 27.8 / 29.5).  Only the table's capacity is
// known on the host, so of fewer than 1024 items one that could take 25 us is never whole: the
// lengths may be anything.  More items are whole whatever they could take: they fill the chip four
// times, so that equal lengths lose by sharing, though uneven ones would gain (us whole / shared;
// 32 sequences, 32 heads of 128, of 300 keys in a table of 8192 positions 32.5 / 43.3, of 1000 92.5 /
// 100.5, of 8000 700 / 705, one of 32000 among 31 of 300 383 / 127; 32/8 heads, 128 sequences of
// 4000 to 8000 524 / 542, of 100 to 8000 220 / 186, 512 of 500 186 / 209).  8 wavefronts a whole
// item: 16 sequences of 1000 keys, 8 heads of 32, 8.4 us, with 4 9.7; 2048 items of 700 keys 103.8
// and 102.6.

PagedWay paged_way(const gm_paged_cache& c, int B, int n, int width, int n_heads, int window, bool packed) {
  PagedWay w;
  const bool f32 = c.dtype == kF32;
  const int G = n_heads / c.heads;
  const int64_t most = static_cast<int64_t>(n) * G;        // rows of a key head of one sequence
  w.many = !f32 && most > kFewRows;
  const int64_t cap = static_cast<int64_t>(width) * c.page_size;
  // (of a packed call, some sequences may be of few rows; over short caches the prompt kernel
  // takes them too, for a launch less: 4 chunks of 100 tokens, 12 heads of 64, of 500 keys 11.2
  // us, with both kernels 12.9)
  w.few = !w.many || (packed && cap > 512);
  w.nset = most > 16 ? 2 : 1;
  const int R = 16 * w.nset;
  PagedPlan& p = w.rows;
  p.G = G;
  p.few = w.many ? kFewRows : 0;
  p.blocks = packed ? 0 : static_cast<int>((most + R - 1) / R);
  // (rows of a packed call lie in at most a block a sequence more than they fill; where
  // sequences of more than a block are another kernel's, in one a sequence)
  p.items = c.heads * (!packed ? p.blocks * B : w.many ? B : static_cast<int>(most / R) + B);
  p.joined = static_cast<int>(std::min<int64_t>(most, R));
  const int64_t keys = window > 0 ? std::min<int64_t>(cap, static_cast<int64_t>(window) + n) : cap;
  const int tile = f32 ? 16 : 32;
  const double item_us = keys * c.head_dim * (f32 ? 8. : 4.) / 46e3, all_us = item_us * p.items * (46e3 / 4.9e6);
  p.wgs = 0;
  w.waves = 8;
  if (p.items > 512 || keys <= 8 * tile) w.waves = 4;
  // (sequences of few rows beside chunks of many: a launch less for up to 7 us more)
  if (p.items < 1024 && (item_us > 25. || item_us > all_us + (w.many ? 12. : 5.))) {
    const int64_t tiles = (keys + tile * 4 - 1) / (tile * 4) * p.items;
    w.waves = tiles >= 512 ? 8 : 4;
    p.wgs = static_cast<int>(tiles >= 512 ? 256 : tiles);
  }
  w.rows_bytes = w.few && p.wgs ? static_cast<uint64_t>(p.wgs) * 2 * R * (c.head_dim + 2) * sizeof(float) : 0;
  return w;
}

}  // namespace

void launch_paged_append(const gm_paged_append_args& a, hipStream_t s) {
  const gm_paged_cache& c = *a.cache;
  const int tokens = a.rows.offsets ? a.rows.n : a.rows.B * a.rows.n;
  // A wavefront a token where tokens are many and a head's threads times heads fill it three
  // times at the most (us with a wavefront / a workgroup a token: bf16, 4000 tokens of 2/2
  // heads of 64 4.6 / 6.7, of 12/12 8.4 / 9.8, of 32/8 heads of 128 17.7 / 18.1; but 16,000 of
  // those in fp16 82.0 / 78.4, 2048 of 32/32 19.5 / 18.0, and 400 of 12/12 heads of 64 4.7 / 3.9).
  const bool small = (a.n_q_heads + 2 * c.heads) * (c.head_dim / 16) <= 192 && tokens >= 1024;
  by_paged_cache(c, [&](auto t, auto hd) {
    typedef decltype(t) T;
    constexpr int HD = decltype(hd)::value;
    if (small)
      hipLaunchKernelGGL((k_paged_append<T, HD, 64>), dim3((tokens + 3) / 4), dim3(256), 0, s, a, c, tokens);
    else
      hipLaunchKernelGGL((k_paged_append<T, HD, 256>), dim3(tokens), dim3(256), 0, s, a, c, tokens);
  });
}

uint64_t paged_attention_workspace(const gm_paged_cache& c, int B, int n, int width, int n_heads, int window, bool packed) {
  const PagedWay w = paged_way(c, B, n, width, n_heads, window, packed);
  // (the two kernels run one after the other)
  const uint64_t many = w.many ? paged_prompt_workspace(c, B, n, width, n_heads, w.few ? kFewRows : 0, packed) : 0;
  return w.rows_bytes > many ? w.rows_bytes : many;
}

void launch_paged_attention(const gm_paged_attention_args& a, hipStream_t s) {
  const gm_paged_cache& c = *a.cache;
  const PagedWay w = paged_way(c, a.rows.B, a.rows.n, a.rows.width, a.n_heads, a.window, a.rows.offsets != nullptr);
  if (w.many) launch_paged_prompt(a, w.few ? kFewRows : 0, s);
  if (!w.few) return;
  const PagedPlan p = w.rows;
  by_paged_cache(c, [&](auto t, auto hd) {
    typedef decltype(t) T;
    constexpr int HD = decltype(hd)::value;
    auto go = [&](auto sets, auto cap, auto waves) {
      constexpr int NSET = decltype(sets)::value, NWV = decltype(waves)::value, UNIT = NWV * (sizeof(T) == 4 ? 16 : 32);
      hipLaunchKernelGGL((k_paged_rows<T, HD, NSET, decltype(cap)::value, NWV>), dim3(p.wgs ? p.wgs : p.items),
                         dim3(64 * NWV), 0, s, a, c, p);
      if (p.wgs)
        hipLaunchKernelGGL((k_paged_join<T, HD, 16 * NSET, UNIT>), dim3(p.wgs, (p.joined + 3) / 4), dim3(256), 0, s,
                           a, c, p);
    };
    auto wide = [&](auto sets, auto cap) {
      if (w.waves == 8) go(sets, cap, std::integral_constant<int, 8>());
      else go(sets, cap, std::integral_constant<int, 4>());
    };
    auto width = [&](auto cap) {
      if (w.nset == 1) wide(std::integral_constant<int, 1>(), cap);
      else wide(std::integral_constant<int, 2>(), cap);
    };
    if (a.scores.softcap > 0.f) width(std::true_type());
    else width(std::false_type());
  });
}

}  // namespace gm
