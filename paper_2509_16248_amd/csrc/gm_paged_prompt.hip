// gm_paged_prompt.hip -- attention of prompts and chunks of prompts over a paged
// KV cache (gm.h, gm_paged_attention), 16-bit types.
#include <math.h>

#include <algorithm>

#include "gm_device.h"
#include "gm_paged.h"

namespace gm {

namespace {

// Row r of key head kvh of a sequence: token r / G, query head kvh * G + r % G, so that the
// heads of a group share a workgroup's keys.
struct PromptPlan {
  int G;
  int blocks;     // blocks of 128 rows of a key head; 0: packed, each sequence has its own
  int most;       // blocks of all sequences at the most
  int few;        // sequences of at most this many rows are another kernel's
  int split;      // keys of a block may be cut into parts
  // Blocks of a sequence from this one on, counted from its last, come the other way round (`blocks`:
  // none do).  Of 257 to 512 items, which run at once, the first 256 have a CU each and the others
  // join them in order: turned round, the shortest of them joins the longest.  Us in order / turned,
  // bf16, one prompt, 32 heads of 128: 1300 tokens 34.9 / 34.6, 1536 39.5 / 37.5, 1900 49.5 / 46.1,
  // 2048 53.8 / 50.1; 24 heads, 2600 tokens 65.2 / 65.0, 12 heads, 4096 tokens 89.9 / 89.4.  More
  // items run one after the other, and lose 1 to 3%.
  int turned;
};

constexpr int kRows = 128, kKeys = 64;   // a workgroup's rows, keys of a tile
constexpr int kSlots = 512;              // workgroups that run at a time, two on a CU
// Tiles a part has at the least, and a table whose calls cut blocks at all, which takes the
// join's launch (parts of 8 / 3 tiles: 4 packed chunks of 713 tokens of 1024, one head of 64, 24.6 /
// 18.8 us; but 600 tokens, 12 heads of 64, whole 12.2, cut 15.5).
constexpr int kLeastTiles = 3, kSplitTiles = 16;

// Parts that items (blocks and key heads) are cut into where they leave slots empty.
__host__ __device__ inline int prompt_cuts(long long items) {
  const long long n = items > 0 && items < kSlots / 2 ? kSlots / items : 1;
  return n < 16 ? static_cast<int>(n) : 16;
}
// The cuts of a call; packed rows' blocks are counted by a wavefront.
__device__ __forceinline__ int prompt_cuts(const gm_paged_attention_args& a, const gm_paged_cache& c, const PromptPlan& p) {
  if (!p.split) return 1;
  int blocks = p.most;
  if (!p.blocks) {
    blocks = 0;
    for (int b = threadIdx.x & 63; b < a.rows.B; b += 64) {
      const int rows = paged_seq(a, c, b).n * p.G;
      blocks += rows > p.few ? (rows + kRows - 1) / kRows : 0;
    }
    blocks = __builtin_amdgcn_readlane(wave_scan(blocks), 63);
  }
  return prompt_cuts(static_cast<long long>(blocks) * c.heads);
}

// A workgroup's block of rows, and the keys it goes through.
struct PromptPlace {
  int b, kvh, qb, split;                 // b = -1: none
  long long item;                        // which (block, key head) of the call
  PagedSeq s;
  int rows;                              // of the sequence's key heads
  int qmin, qmax;                        // positions of the block's first and last row
  int k0, k1, parts;                     // keys, from a multiple of 64; parts that the block has
};
__device__ __forceinline__ PromptPlace prompt_place(const gm_paged_attention_args& a, const gm_paged_cache& c,
                                                    const PromptPlan& p, int block, int kvh, int cuts, int split) {
  PromptPlace w;
  w.kvh = kvh;
  w.split = split;
  w.item = static_cast<long long>(block) * c.heads + kvh;
  int qb;                                // counted from the first row
  if (p.blocks) {
    // later tokens, which see more keys, first; sequences in turn (and PromptPlan::turned)
    int x = block / a.rows.B;
    w.b = block - x * a.rows.B;
    if (x >= p.turned) x = p.turned + p.blocks - 1 - x;
    qb = p.blocks - 1 - x;
    w.s = paged_seq(a, c, w.b);
  } else {
    const int lane = threadIdx.x & 63;
    int before = 0;
    w.b = -1;
    for (int b0 = 0; b0 < a.rows.B; b0 += 64) {
      int nb = 0;
      if (b0 + lane < a.rows.B) {
        const int rows = paged_seq(a, c, b0 + lane).n * p.G;
        nb = rows > p.few ? (rows + kRows - 1) / kRows : 0;
      }
      int sum = nb;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(sum, o, 64);
        if (lane >= o) sum += y;
      }
      const unsigned long long hit = __ballot(block < before + sum && block >= before + sum - nb);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        w.b = b0 + l;
        qb = __builtin_amdgcn_readlane(sum, l) + before - 1 - block;   // (the last block first)
        break;
      }
      before += __builtin_amdgcn_readlane(sum, 63);
    }
    if (w.b < 0) return w;
    w.b = __builtin_amdgcn_readfirstlane(w.b);
    w.s = paged_seq(a, c, w.b);
  }
  w.qb = __builtin_amdgcn_readfirstlane(qb);
  w.rows = w.s.n * p.G;
  const int last = (w.qb + 1) * kRows < w.rows ? (w.qb + 1) * kRows - 1 : w.rows - 1;
  w.qmin = w.s.p0 + w.qb * kRows / p.G;
  w.qmax = w.s.p0 + last / p.G;
  w.k0 = a.window > 0 && w.qmin - a.window + 1 > 0 ? (w.qmin - a.window + 1) & ~(kKeys - 1) : 0;
  w.k1 = w.qmax + 1 < w.s.kend ? w.qmax + 1 : w.s.kend;
  const int tiles = w.k1 > w.k0 ? (w.k1 - w.k0 + kKeys - 1) / kKeys : 0;
  w.parts = 1;
  if (cuts > 1 && tiles >= 2 * kLeastTiles) {
    const int want = tiles / kLeastTiles < cuts ? tiles / kLeastTiles : cuts;
    const int per = (tiles + want - 1) / want;
    w.parts = (tiles + per - 1) / per;
    w.k0 += split * per * kKeys;
    const int end = w.k0 + per * kKeys;
    w.k1 = w.k1 < end ? w.k1 : end;
  }
  return w;
}

template <int HD>
__device__ __forceinline__ float* prompt_part(const gm_paged_attention_args& a, const PromptPlace& w, int cuts, int split) {
  return static_cast<float*>(a.workspace) + (w.item * cuts + split) * kRows * (HD + 2);
}

// One, two or four instructions of 1 KB into LDS, one after the other there and, but for a
// lane's own bytes off[j], in memory.
__device__ __forceinline__ void copy_rows(const char* g, const uint32_t (&off)[1], void* lds) {
  __builtin_amdgcn_global_load_lds(g + off[0], (lds_vptr)lds, 16, 0, 0);
}
__device__ __forceinline__ void copy_rows(const char* g, const uint32_t (&off)[2], void* lds) {
  __builtin_amdgcn_global_load_lds(g + off[0], (lds_vptr)lds, 16, 0, 0);
  __builtin_amdgcn_global_load_lds(g + off[1], (lds_vptr)lds, 16, 1024, 0);
}
__device__ __forceinline__ void copy_rows(const char* g, const uint32_t (&off)[4], void* lds) {
  __builtin_amdgcn_global_load_lds(g + off[0], (lds_vptr)lds, 16, 0, 0);
  __builtin_amdgcn_global_load_lds(g + off[1], (lds_vptr)lds, 16, 1024, 0);
  __builtin_amdgcn_global_load_lds(g + off[2], (lds_vptr)lds, 16, 2 * 1024, 0);
  __builtin_amdgcn_global_load_lds(g + off[3], (lds_vptr)lds, 16, 3 * 1024, 0);
}

constexpr int paged_prompt_waves(int hd) { return hd == 128 ? 2 : hd == 64 ? 3 : 4; }

// Workgroup = 128 query rows of one (sequence, key head), as k_prompt_flash
// (gm_attention_prompt.hip) splits and multiplies: 4 wavefronts x 32 rows, key and value
// tiles of 64 keys double-buffered in LDS, S^T = K Q^T and O^T += V^T P^T on 32x32x16, a
// lane holding 32 scores of one row per tile, the running maximum moved lazily.
// A wavefront copies 16 rows of a tile, which lie in one page (pages are multiples of 16): a
// word per lane holds the tile's 64 table entries, read a tile ahead, one of which gives the
// scalar address, and those that are no page give the tile's holes in a ballot.  Rows past
// the last key repeat it.  (Addresses by lane: 300 vector instructions a tile, 60.6 us for the
// 2048 tokens below; so 52.9.)
// LDS is read ahead of the products by hand: K two k steps, V one of 16 keys (left to the
// compiler each K operand's read waits for the one before: 2 us more).
// Probabilities are rounded to T for the second product (half a step of each, up to 2^-8 or
// 2^-11 of it; their sum takes them unrounded): its operands are 16-bit.
// A hidden key has probability 0, but 0 times an Inf or NaN value is NaN in the matrix
// product: rows whose sums came out not finite are computed again by paged_row, which skips
// hidden keys.
// Measured, bf16, 32 heads of 128, launches one after the other: 2048 tokens 48 to 51 us (700
// TFLOP/s; capped 57, biased 56), 4 x 2048 with 8 key heads 154 (890), 8192 tokens 530 (1040; a
// large matrix product reaches 1197), 512 tokens behind 7680 85 (770).  What bounds it: a SIMD's
// two wavefronts keep the matrix cores busy 49% and the vector units 42% of the time that CUs
// hold work, each wavefront's own chain of instructions taking the rest.  Not faster: the next
// tile's scores beside this one's probabilities in one wavefront (the registers of two score
// tiles spill, 2 x slower; at one wavefront per SIMD without spilling 1.6 x), halves of a tile
// in turn (54.7 us against 52.9), more than one running sum or maximum, wavefront priorities.
template <typename T, int HD, bool CAP, bool BIAS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(paged_prompt_waves(HD), paged_prompt_waves(HD))))
void k_paged_prompt(gm_paged_attention_args a, gm_paged_cache c, PromptPlan plan) {
  constexpr int KB = kKeys, NW = 4;
  typedef typename Mfma32A<T>::vec vec;
  constexpr int KS = HD / 16;                 // k steps of S^T (head dim)
  constexpr int CB = HD / 32;                 // 32-channel blocks of O^T
  constexpr int CPR = HD / 8;                 // 16-byte chunks per key row
  constexpr int RPL = 16 / CPR;               // key rows per 256 bytes
  constexpr int RPI = 64 / CPR;               // key rows per 1 KB copy instruction
  constexpr int LPW = KB / RPI / NW;          // copy instructions per wavefront, tile and operand
  constexpr int TILE = KB * HD;
  __shared__ __attribute__((aligned(1024))) T lds[4 * TILE];   // K of two stages, V of two

  // heads fastest: the blocks of a key head come to one XCD where the heads are a
  // multiple of 8
  const int cuts = prompt_cuts(a, c, plan);
  int x = blockIdx.x;
  const int kvh = x % c.heads;
  x /= c.heads;
  if (x >= plan.most * cuts) return;
  const PromptPlace w = prompt_place(a, c, plan, x / cuts, kvh, cuts, x % cuts);
  if (w.b < 0 || w.split >= w.parts) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l32 = lane & 31, h2 = lane >> 5;
  const int rw0 = w.qb * kRows + wave * 32;   // first row of this wavefront
  const bool some = rw0 < w.rows;
  const int rlast = rw0 + 31 < w.rows ? rw0 + 31 : w.rows - 1;
  // positions of its first and last; a wavefront without rows copies, and skips every tile (bf16, 4
  // sequences of 6000 keys, 32/8 heads of 128, 160 rows 46.3 -> 44.4 us, 36 rows 33.2 -> 32.7)
  const int wmin = w.s.p0 + rw0 / plan.G, wmax = some ? w.s.p0 + rlast / plan.G : -1;
  const int r = rw0 + l32, rc = r < w.rows ? r : w.rows - 1;
  const int qi = rc / plan.G, h = kvh * plan.G + rc - qi * plan.G;
  const int qpos = w.s.p0 + qi;
  const int window = a.window > 0 ? a.window : 1 << 30;
  const int lg = 31 - __builtin_clz(c.page_size), in_page = c.page_size - 1;
  const int32_t* table = a.rows.table + w.b * a.rows.table_stride;
  const int kend = w.k1, last_key = kend - 1, last_page = a.rows.width - 1;

  vec qf[KS];
  {
    const T* qp = paged_row_at<const T>(a.q, a.rows, w.b, w.s.row0, qi, h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const vec*>(qp + 16 * ks + 8 * h2);
  }
  const float c2 = CAP ? a.scores.scale * (2.f * kPagedLog2e) / a.scores.softcap : a.scores.scale * kPagedLog2e;
  const float capc = a.scores.softcap * kPagedLog2e;
  const float slope2 = BIAS ? a.scores.slopes[h] * -kPagedLog2e : 0.f;
  constexpr bool LOG2 = CAP || BIAS;          // scores are in log2 units before their maximum is taken

  float mrun = -INFINITY, lrun = 0.f;
  f32x16 oacc[CB];
#pragma unroll
  for (int e = 0; e < CB; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[e][i] = 0.f;

  // the table entry of key kb + lane
  auto entries = [&](int kb) {
    const int at = (kb + lane) >> lg;
    return table[at < last_page ? at : last_page];
  };
  // swizzles: chunk e of key row r sits at chunk position e ^ f(r) (k_flash)
  const int cr = lane / CPR, cpos = lane % CPR;
  // A wavefront's rows of a tile, 16 of them, lie in one page.  A lane's bytes from the first
  // row of a copy instruction: of K for each, of V the same for all.
  static_assert(LPW * RPI == 16 && RPI * HD * 2 == 1024, "a wavefront copies 16 rows, 1 KB at a time");
  static_assert(RPI / RPL % (CPR / 4) == 0, "V's swizzle is the same for every copy instruction");
  uint32_t koff[LPW];
#pragma unroll
  for (int j = 0; j < LPW; ++j)
    koff[j] = 2 * (cr * HD + 8 * (cpos ^ (((wave * LPW + j) * RPI + cr) / RPL % CPR)));
  const uint32_t voff = 2 * (cr * HD + 8 * (cpos ^ 4 * (cr / RPL % (CPR / 4))));
  const int64_t page_bytes = static_cast<int64_t>(c.heads) * c.page_size * HD * 2;
  const char* kbase = static_cast<const char*>(c.k) + static_cast<int64_t>(kvh) * c.page_size * HD * 2;
  const char* vbase = static_cast<const char*>(c.v) + static_cast<int64_t>(kvh) * c.page_size * HD * 2;
  // the tile at kb, whose entries are ids; its keys that are in no hole are returned
  auto issue = [&](int kb, int ids, T* dst) {
    const bool ok = static_cast<unsigned>(ids) < static_cast<unsigned>(c.pages);
    const int id = ok ? ids : 0, row = wave * 16;
    T *dk = dst + row * HD, *dv = dk + 2 * TILE;
    if (kb + KB <= kend) {
      const int64_t at = __builtin_amdgcn_readlane(id, row) * page_bytes + ((kb + row) & in_page) * (HD * 2);
      copy_rows(kbase + at, koff, dk);
      const uint32_t same[LPW] = {};
      copy_rows(vbase + at + voff, same, dv);
    } else {
      // (rows past the last key repeat it; a wavefront's rows that all lie past it those before)
      const int first = kb + row < (last_key & ~15) ? kb + row : last_key & ~15;
      const int64_t at = __builtin_amdgcn_readlane(id, first - kb) * page_bytes + (first & in_page) * (HD * 2);
#pragma unroll
      for (int j = 0; j < LPW; ++j) {
        const int past = first + j * RPI + cr - last_key, back = past > 0 ? past * HD * 2 : 0;
        dma16(kbase + at + (static_cast<int>(koff[j]) + j * 1024 - back), dk + j * RPI * HD);
        dma16(vbase + at + (static_cast<int>(voff) + j * 1024 - back), dv + j * RPI * HD);
      }
    }
    return __ballot(ok);
  };
  const int kswz = (l32 / RPL) % CPR;
  const int g = lane >> 4, e4 = (lane & 15) >> 2, q4 = lane & 3;
  const int vrow = 4 * (g >> 1) + e4;
  const int vswz4 = (vrow / RPL) % (CPR / 4);
  const int vsub = 2 * (g & 1) + (q4 >> 1);
  const int vin = 4 * (q4 & 1);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_vptr)lds));
  uint32_t kaddr[KS], vaddr[CB];              // in stage 0
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = lds0 + 2 * (l32 * HD + 8 * ((2 * ks + h2) ^ kswz));
#pragma unroll
  for (int e = 0; e < CB; ++e) vaddr[e] = lds0 + 2 * (2 * TILE + vrow * HD + 8 * (4 * (e ^ vswz4) + vsub) + vin);

  unsigned long long there[2] = {0, 0};       // keys of the stages' tiles that are in no hole
  int ids = 0;                                // entries of the tile after the next
  // one key tile from stage BUF (the other stage receives the next one)
  auto tile = [&](auto BUF, int kb) {
    constexpr int buf = decltype(BUF)::value, STAGE = 2 * buf * TILE;   // bytes of it
    T* other = lds + (buf ^ 1) * TILE;
    wait_vmcnt0();                            // this wavefront's copies of the tile landed
    __syncthreads();
    if (kb + KB < kend) {
      there[buf ^ 1] = issue(kb + KB, ids, other);
      ids = entries(kb + 2 * KB);
    }
    // no key of the tile is seen by this wavefront's rows
    if (kb > wmax || kb + KB - 1 <= wmin - window) return;
    const unsigned long long bits = there[buf] & (kend - kb >= KB ? ~0ull : (1ull << (kend - kb)) - 1);
    // ---- S^T = K Q^T: two 32-key blocks
    f32x16 sacc[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 16; ++i) sacc[kk][i] = 0.f;
    // (the K operands of two k steps on their way while one multiplies)
    u32x4 kf[3][2];
    auto kread = [&](int ks) {
      kf[ks % 3][0] = lds_read16<STAGE>(kaddr[ks]);
      kf[ks % 3][1] = lds_read16<STAGE + 64 * HD>(kaddr[ks]);
    };
    auto kmul = [&](int ks) {
      sacc[0] = Mfma32A<T>::run(__builtin_bit_cast(vec, kf[ks % 3][0]), qf[ks], sacc[0]);
      sacc[1] = Mfma32A<T>::run(__builtin_bit_cast(vec, kf[ks % 3][1]), qf[ks], sacc[1]);
    };
    kread(0);
    kread(1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) {
        kread(ks + 2);
        lgkm_wait16<4>(kf[ks % 3]);
      } else if (ks + 1 < KS) {
        lgkm_wait16<2>(kf[ks % 3]);
      } else {
        lgkm_wait16<0>(kf[ks % 3]);
      }
      kmul(ks);
    }
    // ---- capped scores, in log2 units
    if constexpr (CAP) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(sacc[kk][i] * c2) + 1.f;
          sacc[kk][i] = fmaf(-2.f * capc, __builtin_amdgcn_rcpf(e), capc);
        }
    }
    if constexpr (BIAS) {
      const float dist = static_cast<float>(qpos - kb - 4 * h2);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sacc[kk][i] = fmaf(slope2, dist - static_cast<float>(32 * kk + 8 * (i >> 2) + (i & 3)),
                             CAP ? sacc[kk][i] : sacc[kk][i] * c2);
    }
    // ---- masks
    if (bits != ~0ull || kb + KB - 1 > wmin || kb <= wmax - window) {
      const int n = qpos + 1 - kb, low = n - window;   // keys [low, n) of the tile
      unsigned long long vis = bits & (n >= KB ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1);
      vis &= low <= 0 ? ~0ull : low >= KB ? 0ull : ~((1ull << low) - 1);
      vis >>= 4 * h2;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sacc[kk][i] = (vis >> (32 * kk + 8 * (i >> 2) + (i & 3))) & 1ull ? sacc[kk][i] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sacc[kk][i]);
    float mt = LOG2 ? mx : mx * c2;
    if (__ballot(mt > mrun + kTau)) {          // move the maximum (wavefront-uniform)
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
      const float mnew = fmaxf(mrun, mt);
      const float alpha = mnew == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mrun - mnew);
      lrun *= alpha;
#pragma unroll
      for (int e = 0; e < CB; ++e) oacc[e] *= alpha;
      mrun = mnew;
    }
    const float msub = mrun == -INFINITY ? 0.f : mrun - kWeightUp<T>;
    // ---- O^T += V^T P^T: four 16-key steps; the V^T operands of step k2 + 1 are read
    // while step k2 multiplies, those of the first while the probabilities are computed
    vec pb[4];
    u32x2 vf[2][CB][2];
    auto vread = [&](auto K2, u32x2 (&dst)[CB][2]) {
      constexpr int k2 = decltype(K2)::value;
#pragma unroll
      for (int e = 0; e < CB; ++e) {
        dst[e][0] = lds_read_tr16<STAGE + (16 * k2) * HD * 2>(vaddr[e]);
        dst[e][1] = lds_read_tr16<STAGE + (16 * k2 + 8) * HD * 2>(vaddr[e]);
      }
    };
    auto vmul = [&](int k2, u32x2 (&src)[CB][2]) {
#pragma unroll
      for (int e = 0; e < CB; ++e) {
        u32x4 v;
        v[0] = src[e][0][0]; v[1] = src[e][0][1]; v[2] = src[e][1][0]; v[3] = src[e][1][1];
        oacc[e] = Mfma32A<T>::run(__builtin_bit_cast(vec, v), pb[k2], oacc[e]);
      }
    };
    vread(std::integral_constant<int, 0>(), vf[0]);
    // ---- probabilities, their sum, and P^T as 16-bit B operands
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s0 = sacc[kk][8 * hf + 2 * j], s1 = sacc[kk][8 * hf + 2 * j + 1];
          const float p0 = __builtin_amdgcn_exp2f(LOG2 ? s0 - msub : fmaf(s0, c2, -msub));
          const float p1 = __builtin_amdgcn_exp2f(LOG2 ? s1 - msub : fmaf(s1, c2, -msub));
          lrun += p0 + p1;
          v[j] = pack2<T>(p0, p1);
        }
        pb[2 * kk + hf] = __builtin_bit_cast(vec, v);
      }
    }
    vread(std::integral_constant<int, 1>(), vf[1]);
    lgkm_wait<2 * CB>(&vf[0][0][0], 2 * CB);
    vmul(0, vf[0]);
    vread(std::integral_constant<int, 2>(), vf[0]);
    lgkm_wait<2 * CB>(&vf[1][0][0], 2 * CB);
    vmul(1, vf[1]);
    vread(std::integral_constant<int, 3>(), vf[1]);
    lgkm_wait<2 * CB>(&vf[0][0][0], 2 * CB);
    vmul(2, vf[0]);
    lgkm_wait<0>(&vf[1][0][0], 2 * CB);
    vmul(3, vf[1]);
  };
  if (w.k0 < kend) {
    there[0] = issue(w.k0, entries(w.k0), lds);
    ids = entries(w.k0 + KB);
    for (int kb = w.k0;; kb += 2 * KB) {
      tile(std::integral_constant<int, 0>(), kb);
      if (kb + KB >= kend) break;
      tile(std::integral_constant<int, 1>(), kb + KB);
      if (kb + 2 * KB >= kend) break;
    }
  }
  // ---- normalise and store: lane holds channels 32 e + 8 i + 4 (lane / 32) + j of its row
  const float L = lrun + __shfl_xor(lrun, 32, 64);
  float odd = 0.f * L;
#pragma unroll
  for (int e = 0; e < CB; ++e)
#pragma unroll
    for (int i = 0; i < 16; ++i) odd = fmaf(oacc[e][i], 0.f, odd);
  const unsigned long long odd_lanes = __ballot(odd != 0.f);   // (NaN != 0)
  uint32_t again = static_cast<uint32_t>(odd_lanes) | static_cast<uint32_t>(odd_lanes >> 32);
  float* part = w.parts > 1 ? prompt_part<HD>(a, w, cuts, w.split) + wave * 32 * (HD + 2) : nullptr;
  if (r < w.rows && !(again >> l32 & 1)) {
    const float inv = L > 0.f ? 1.f / L : 0.f;
    if (part) {
      float* o = part + l32 * (HD + 2);
      if (h2 == 0) *reinterpret_cast<f32x2*>(o) = f32x2{mrun, L * kWeightDown<T>};
#pragma unroll
      for (int e = 0; e < CB; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            *reinterpret_cast<f32x2*>(o + 2 + 32 * e + 8 * i + 4 * h2 + 2 * j) =
                f32x2{oacc[e][4 * i + 2 * j] * inv, oacc[e][4 * i + 2 * j + 1] * inv};
    } else {
      T* out = paged_row_at<T>(a.out, a.rows, w.b, w.s.row0, qi, h);
#pragma unroll
      for (int e = 0; e < CB; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x2 r2;
          r2[0] = pack2<T>(oacc[e][4 * i] * inv, oacc[e][4 * i + 1] * inv);
          r2[1] = pack2<T>(oacc[e][4 * i + 2] * inv, oacc[e][4 * i + 3] * inv);
          *reinterpret_cast<u32x2*>(out + 32 * e + 8 * i + 4 * h2) = r2;
        }
    }
  }
  for (; __builtin_expect(again != 0, 0); again &= again - 1) {
    const int j = __builtin_ctz(again), row = rw0 + j;
    if (row >= w.rows) break;
    const int i = row / plan.G, hh = kvh * plan.G + row - i * plan.G;
    T* out = paged_row_at<T>(a.out, a.rows, w.b, w.s.row0, i, hh);
    const f32x2 ml = paged_row<T, HD>(a, c, w.s, w.b, hh, i, w.k0, w.k1, [&](int ch, float v) {
      if (part) part[j * (HD + 2) + 2 + ch] = v;
      else out[ch] = from_f32<T>(v);
    });
    if (part && lane == 0) {
      part[j * (HD + 2)] = ml[0];
      part[j * (HD + 2) + 1] = ml[1];
    }
  }
}

// The parts of a block's rows joined in order of their keys, a wavefront a row; 4 rows at a
// time of at most kSlots / 2 items by a grid that fits the chip.
constexpr int kJoins = 2048;
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_paged_prompt_join(gm_paged_attention_args a, gm_paged_cache c, PromptPlan plan) {
  const int cuts = prompt_cuts(a, c, plan);
  if (cuts == 1) return;
  constexpr int64_t STEP = kRows * (HD + 2);
  constexpr int CL = (HD + 63) / 64, U = 4;    // channels of a lane, parts loaded together
  const int lane = threadIdx.x & 63;
  for (int x = blockIdx.x; x < kSlots / cuts * (kRows / 4); x += gridDim.x) {
    const int item = x / (kRows / 4), row = x % (kRows / 4) * 4 + (threadIdx.x >> 6);
    const int block = item / c.heads, kvh = item - block * c.heads;
    if (block >= plan.most) return;
    const PromptPlace w = prompt_place(a, c, plan, block, kvh, cuts, 0);
    if (w.b < 0) return;
    const int r = w.qb * kRows + row;
    if (w.parts < 2 || r >= w.rows) continue;
    const float* part = prompt_part<HD>(a, w, cuts, 0) + row * (HD + 2);
    float v[U][CL];
    auto fetch = [&](int p0) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < CL; ++e)
          v[u][e] = p0 + u < w.parts && lane + 64 * e < HD ? part[(p0 + u) * STEP + 2 + lane + 64 * e] : 0.f;
    };
    fetch(0);
    const bool on = lane < w.parts;
    const float m = on ? part[lane * STEP] : -INFINITY, l = on ? part[lane * STEP + 1] : 0.f;
    const float M = wave_max(m);
    float f = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - M);
    const float F = wave_sum(f);
    f = f == 0.f ? 0.f : f / F;
    float o[CL] = {};
    for (int p0 = 0; p0 < w.parts; p0 += U) {
      if (p0) fetch(p0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fp = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), p0 + u));
#pragma unroll
        for (int e = 0; e < CL; ++e) o[e] += fp == 0.f ? 0.f : fp * v[u][e];
      }
    }
    const int i = r / plan.G;
    T* out = paged_row_at<T>(a.out, a.rows, w.b, w.s.row0, i, kvh * plan.G + r - i * plan.G);
#pragma unroll
    for (int e = 0; e < CL; ++e)
      if (lane + 64 * e < HD) out[lane + 64 * e] = from_f32<T>(o[e]);
  }
}

PromptPlan prompt_plan(const gm_paged_cache& c, int B, int n, int width, int n_heads, bool packed, int few) {
  PromptPlan p;
  p.G = n_heads / c.heads;
  p.few = few;
  const int64_t rows = static_cast<int64_t>(n) * p.G;      // of a key head
  p.blocks = packed ? 0 : static_cast<int>((rows + kRows - 1) / kRows);
  // (packed: at most a block more than they fill for each sequence of more than `few` rows)
  p.most = packed ? static_cast<int>(rows / kRows + std::min<int64_t>(B, rows / (few + 1))) : p.blocks * B;
  const int64_t tiles = static_cast<int64_t>(width) * c.page_size / kKeys;
  // (of packed rows, those that must lie in blocks)
  const int64_t least = packed ? std::max<int64_t>(0, rows - static_cast<int64_t>(B) * few + kRows - 1) / kRows : p.most;
  const int64_t pairs = static_cast<int64_t>(B) * c.heads, items = p.blocks * pairs;
  p.turned = p.blocks;
  if (items > kSlots / 2 && items <= kSlots) p.turned = static_cast<int>((kSlots / 2 + pairs - 1) / pairs);
  p.split = tiles >= kSplitTiles && prompt_cuts(std::max<int64_t>(least, 1) * c.heads) > 1;
  return p;
}

}  // namespace

uint64_t paged_prompt_workspace(const gm_paged_cache& c, int B, int n, int width, int n_heads, int few, bool packed) {
  const PromptPlan p = prompt_plan(c, B, n, width, n_heads, packed, few);
  // (where blocks are cut up, their parts fill the slots at the most)
  return p.split ? static_cast<uint64_t>(kSlots) * kRows * (c.head_dim + 2) * sizeof(float) : 0;
}

void launch_paged_prompt(const gm_paged_attention_args& a, int few, hipStream_t s) {
  const gm_paged_cache& c = *a.cache;
  const PromptPlan p = prompt_plan(c, a.rows.B, a.rows.n, a.rows.width, a.n_heads, a.rows.offsets != nullptr, few);
  // (whole multiples of the heads)
  const unsigned items = static_cast<unsigned>(p.most) * c.heads, slots = (kSlots + c.heads - 1) / c.heads * c.heads;
  const unsigned grid = p.split && items < slots ? slots : items;
  const bool cap = a.scores.softcap > 0.f, bias = a.scores.slopes;
  const std::true_type yes;
  const std::false_type no;
  by_paged_cache(c, [&](auto t, auto hd) {
    typedef decltype(t) T;
    if constexpr (!std::is_same<T, float>::value) {
      constexpr int HD = decltype(hd)::value;
      auto go = [&](auto cp, auto bi) {
        hipLaunchKernelGGL((k_paged_prompt<T, HD, decltype(cp)::value, decltype(bi)::value>),
                           dim3(grid), dim3(256), 0, s, a, c, p);
      };
      if (cap && bias) go(yes, yes);
      else if (cap) go(yes, no);
      else if (bias) go(no, yes);
      else go(no, no);
      if (p.split) hipLaunchKernelGGL((k_paged_prompt_join<T, HD>), dim3(kJoins), dim3(256), 0, s, a, c, p);
    }
  });
}

}  // namespace gm
