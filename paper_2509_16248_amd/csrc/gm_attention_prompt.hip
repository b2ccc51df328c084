// gm_attention_prompt.hip -- attention over whole prompts with modified scores
// (gm.h, gm_attention): a tanh cap, a bias by distance, and key, document and
// prefix masks next to the causal one; query heads may share key heads.
#include <math.h>

#include <type_traits>

#include "gm_device.h"
#include "gm_flash.h"
#include "gm_ops.h"

namespace gm {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// One query by one wavefront, a key per lane: two passes over the keys, the largest
// score and the weights' sum, then the output, of weights that add up to 1, so that
// it overflows only where it has to.  A hidden key is skipped, so that nothing its
// value holds can reach the sums.
template <typename T, int HD>
__device__ __forceinline__ void prompt_row(const gm_prompt_attention& a, int b, int h, int i) {
  constexpr int CL = (HD + 63) / 64;   // channels per lane
  const int lane = threadIdx.x & 63;
  const int kvh = h / (a.n_heads / a.kv_heads);
  const T* q = static_cast<const T*>(a.q.p) + b * a.q.batch + i * a.q.token + h * a.q.head;
  const T* kb = static_cast<const T*>(a.k.p) + b * a.k.batch + kvh * a.k.head;
  const T* vb = static_cast<const T*>(a.v.p) + b * a.v.batch + kvh * a.v.head;
  const int32_t* mk = a.key_mask ? a.key_mask + static_cast<long long>(b) * a.Sk : nullptr;
  const int32_t* kd = a.q_doc ? a.k_doc + static_cast<long long>(b) * a.Sk : nullptr;
  const int qd = a.q_doc ? a.q_doc[static_cast<long long>(b) * a.Sq + i] : 0;
  const float slope = a.scores.slopes ? a.scores.slopes[h] : 0.f;
  const int qpos = i + a.q_offset;
  int kend = a.Sk;
  if (a.causal) {
    const int pre = a.prefix ? a.prefix[b] : 0;
    const int last = qpos + 1 > pre ? qpos + 1 : pre;
    kend = kend < last ? kend : last;
  }
  auto visible = [&](int j) { return j < kend && (!mk || mk[j] != 0) && (!kd || kd[j] == qd); };
  auto score = [&](int j) {
    const T* k = kb + j * a.k.token;
    float s = 0.f;
#pragma unroll 4
    for (int c = 0; c < HD; ++c) s = fmaf(to_f32(q[c]), to_f32(k[c]), s);
    return modify_score(s * a.scores.scale, a.scores.softcap, slope, fabsf(static_cast<float>(qpos - j)));
  };
  float m = -INFINITY, l = 0.f;
  for (int j0 = 0; j0 < kend; j0 += 64) {
    if (!visible(j0 + lane)) continue;
    const float x = score(j0 + lane);
    if (x == -INFINITY) continue;
    const float mn = fmaxf(m, x);
    l = (m == -INFINITY ? l : l * expf(m - mn)) + expf(x - mn);   // (a NaN stays)
    m = mn;
  }
  const float M = wave_max(m);
  l = wave_sum(m == -INFINITY ? l : l * expf(m - M));
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float o[CL] = {};
  for (int j0 = 0; j0 < kend; j0 += 64) {
    const bool ok = visible(j0 + lane);
    float p = 0.f;
    if (ok) {
      const float x = score(j0 + lane);
      p = x == -INFINITY ? 0.f : expf(x - M) * inv;
    }
    const unsigned long long on = __ballot(ok);
    for (int t = 0; t < 64 && j0 + t < kend; ++t) {
      const float pt = __shfl(p, t, 64);
      if (!(on >> t & 1)) continue;
      const T* v = vb + (j0 + t) * a.v.token;
#pragma unroll
      for (int c = 0; c < CL; ++c)
        if (lane + 64 * c < HD) o[c] = fmaf(pt, to_f32(v[lane + 64 * c]), o[c]);
    }
  }
  T* out = static_cast<T*>(a.out.p) + b * a.out.batch + i * a.out.token + h * a.out.head;
#pragma unroll
  for (int c = 0; c < CL; ++c)
    if (lane + 64 * c < HD) out[lane + 64 * c] = from_f32<T>(l == 0.f ? 0.f : o[c]);
}

// ------------------------------------------------------------ fp32
// Workgroup = 32 queries of one (sequence, head), as k_attn_f32 (gm_attention.hip)
// splits and multiplies: its 4 wavefronts take the tiles of 32 keys in turn, each with
// an online softmax of its own, and are merged in LDS; S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_32x32x2_f32 with operands straight from global memory, a lane holding 16
// scores of one query.  What each lane's query may see of a tile is settled first, and
// a tile that shows no query anything is not loaded.  Queries whose sums came out not
// finite are computed again by prompt_row: a hidden key's weight is 0, but its product
// with an Inf or NaN value is not.
template <int HD, bool CAP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 3)))
void k_prompt_f32(gm_prompt_attention a) {
  constexpr int NC = HD / 8, CB = HD / 32, NW = 4;
  typedef float f32x4a __attribute__((ext_vector_type(4)));
  __shared__ float s_m[NW][32], s_l[NW][32];
  __shared__ float s_o[NW][HD][33];
  __shared__ uint32_t s_odd[NW];
  // order as in k_prompt_flash: query blocks outermost, heaviest first
  const int nqb = (a.Sq + 31) / 32, P = a.B * a.n_heads, blk = blockIdx.x / P, pair = blockIdx.x - blk * P;
  const int qb = a.causal ? nqb - 1 - blk : blk;
  const int b = pair / a.n_heads, hp = pair - b * a.n_heads;
  const int kvh = hp % a.kv_heads, h = kvh * (a.n_heads / a.kv_heads) + hp / a.kv_heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l32 = lane & 31, g = lane >> 5;
  const int Sq = a.Sq, Sk = a.Sk, q0 = qb * 32, qi = q0 + l32, qpos = qi + a.q_offset;
  const int qc = qi < Sq ? qi : Sq - 1;
  const float* q = static_cast<const float*>(a.q.p) + b * a.q.batch + qc * a.q.token + h * a.q.head + 4 * g;
  const float* kb = static_cast<const float*>(a.k.p) + b * a.k.batch + kvh * a.k.head;
  const float* vb = static_cast<const float*>(a.v.p) + b * a.v.batch + kvh * a.v.head;
  const int32_t* mk = a.key_mask ? a.key_mask + static_cast<long long>(b) * Sk : nullptr;
  const int32_t* kd = a.q_doc ? a.k_doc + static_cast<long long>(b) * Sk : nullptr;
  const int qd = a.q_doc ? a.q_doc[static_cast<long long>(b) * Sq + qc] : 0;
  // scores in log2 units
  const float scale = CAP ? a.scores.scale / a.scores.softcap : a.scores.scale * kLog2e;
  const float capc = a.scores.softcap * kLog2e;
  const float slope = a.scores.slopes ? a.scores.slopes[h] * kLog2e : 0.f;
  const int pre = a.causal && a.prefix ? a.prefix[b] : 0;
  int kend = Sk;                               // keys this lane's query may see end here
  if (a.causal) {
    kend = qpos + 1 > pre ? qpos + 1 : pre;
    kend = kend < Sk ? kend : Sk;
  }
  int ktop = Sk;                               // and those of the workgroup's queries here
  if (a.causal) {
    ktop = q0 + 32 + a.q_offset > pre ? q0 + 32 + a.q_offset : pre;
    ktop = ktop < Sk ? ktop : Sk;
  }
  f32x4a qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const f32x4a*>(q + 8 * c);
  f32x16 o[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  for (int k0 = 32 * wave; k0 < ktop; k0 += 32 * NW) {
    uint32_t vis = 0;                          // bit e: score e's key is visible
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int key = k0 + 8 * (e / 4) + 4 * g + e % 4;
      bool ok = key < kend;
      const int kc = key < Sk ? key : Sk - 1;
      if (mk) ok = ok && mk[kc] != 0;
      if (kd) ok = ok && kd[kc] == qd;
      vis |= (ok ? 1u : 0u) << e;
    }
    if (__ballot(vis != 0) == 0) continue;
    const int kr = k0 + l32 < Sk ? k0 + l32 : Sk - 1;
    const float* k = kb + kr * a.k.token + 4 * g;
    f32x4a kf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) kf[c] = *reinterpret_cast<const f32x4a*>(k + 8 * c);
    // V rows, 32 channels at a time, one step ahead of the products
    float vf[2][16];
    auto fetch_v = [&](int c, float (&dst)[16]) {
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const int key = k0 + 8 * (t / 4) + 4 * g + t % 4;
        dst[t] = vb[(key < Sk ? key : Sk - 1) * a.v.token + l32 + 32 * c];
      }
    };
    fetch_v(0, vf[0]);
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[c][r], qf[c][r], s, 0, 0, 0);
    float top = m;
    const float dist = static_cast<float>(qpos - k0 - 4 * g);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float y = s[e] * scale;
      if constexpr (CAP) y = capc * tanhf(y);
      y = fmaf(-slope, fabsf(dist - static_cast<float>(8 * (e / 4) + e % 4)), y);
      s[e] = vis >> e & 1 ? y : -INFINITY;
      top = fmaxf(top, s[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float corr = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);   // (m = -inf: 0)
    const float msub = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] - msub);
      sum += s[e];
    }
    l = l * corr + sum;
    m = top;
#pragma unroll
    for (int c = 0; c < CB; ++c) {
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][e] *= corr;
      if (c + 1 < CB) fetch_v(c + 1, vf[(c + 1) % 2]);
#pragma unroll
      for (int t = 0; t < 16; ++t) o[c] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[c % 2][t], s[t], o[c], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 32, 64);
  float odd = 0.f * l;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) odd = fmaf(o[c][e], 0.f, odd);
  const unsigned long long odd_lanes = __ballot(odd != 0.f);   // (NaN != 0)
  if (lane == 0) s_odd[wave] = static_cast<uint32_t>(odd_lanes) | static_cast<uint32_t>(odd_lanes >> 32);
  if (g == 0) {
    s_m[wave][l32] = m;
    s_l[wave][l32] = l;
  }
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) s_o[wave][32 * c + 8 * (e / 4) + 4 * g + e % 4][l32] = o[c][e];
  __syncthreads();
  const uint32_t again = s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3];
  for (int e = threadIdx.x; e < 32 * HD; e += 256) {
    const int c = e % HD, i = e / HD;
    if (q0 + i >= Sq) break;
    if (again >> i & 1) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, s_m[w][i]);
    float L = 0.f, O = 0.f, f[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      f[w] = s_m[w][i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][i] - M);
      L += s_l[w][i] * f[w];
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;   // (before the sum, which might pass fp32)
#pragma unroll
    for (int w = 0; w < NW; ++w) O += s_o[w][c][i] * (f[w] * inv);
    static_cast<float*>(a.out.p)[b * a.out.batch + (q0 + i) * a.out.token + h * a.out.head + c] = O;
  }
  if (__builtin_expect(again != 0, 0))
    for (int i = wave; i < 32; i += NW)
      if ((again >> i & 1) && q0 + i < Sq) prompt_row<float, HD>(a, b, h, q0 + i);
}

template <int HD>
void prompt_f32(const gm_prompt_attention& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.Sq + 31) / 32) * a.n_heads * a.B), block(256);
  if (a.scores.softcap > 0.f) hipLaunchKernelGGL((k_prompt_f32<HD, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_prompt_f32<HD, false>), grid, block, 0, s, a);
}

// ------------------------------------------------------------ 16-bit
// 32 bits of four consecutive int32, at any 4-byte address.
typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kTiles = 2048;      // key tiles a workgroup keeps marks for (131072 keys)

// Workgroup = 128 queries of one (sequence, head), as k_flash (gm_attention.hip)
// splits and multiplies: 4 wavefronts x 32 queries, key and value tiles of 64 keys
// double-buffered in LDS, S^T = K Q^T and O^T += V^T P^T on 32x32x16, a lane
// holding 32 scores of one query per tile, the running maximum moved lazily.
// What the scores go through instead:
//  CAP   softcap tanh(x / softcap) = C - 2 C / (exp2(x c2) + 1) in log2 units, C =
//        softcap log2(e): two transcendental and three other instructions
//  BIAS  a subtraction, a multiplication and an fma (after a cap: a subtraction and an
//        fma).  It is added after the scale: slope / scale, from which the products' sums
//        could start, overflows under tiny scales, and what is added to far distances in
//        units of q.k is rounded at every step of the sums.
//  masks a 64-bit word per lane and tile: key mask (a ballot of wavefront 0), causal
//        and prefix bounds (shifts) and documents (32 comparisons where the tile or
//        the wavefront's queries hold more than one); none at all for a tile that is
//        open to every query of the wavefront.
// Tiles without a visible key for the workgroup are not fetched: with a key mask or
// documents every workgroup first reads them all and marks the tiles that hold an
// unmasked key whose document lies in the range of its queries' (any order of documents
// is right; packed ones in order skip nearly all others), and those of one document
// without a masked key, which need no further look: a lane sees all of such a tile or
// nothing.  For the others wavefront 0 fetches mask and documents with the tile.
// SPARSE (masks or documents given) holds all of that; without it the kernel is half as
// long, which 8192 tokens in rows of 128, causal, feel in 57.5 against 46.5 us.
// Probabilities are rounded to T for the second product (half a step of each, up to 2^-8
// or 2^-11 of it; their sum takes them unrounded): its operands are 16-bit.
// Measured, launches one after the other, 32 heads of 128, bf16, causal: 2048 tokens 56.7
// us (606 TFLOP/s), capped 65.9, biased 60.0, both 69.6; without the causal mask 75.2 us
// (914 TFLOP/s), capped 94.2; 8192 tokens and 8 key heads 535 us (1028 TFLOP/s), in 7 equal
// documents 171 (459: tiles that straddle two documents, and workgroups of unequal
// length).  What bounds a short row is that its heaviest workgroup has twice the average
// (the capped 2048 tokens: CUs hold work 71% of the time) and a tile's chain of dependent
// steps, in which at two wavefronts per SIMD the vector units work 60% of that time and
// the matrix cores 29%; vector instructions taken out of the cap (a polynomial) changed
// nothing.
// A hidden key has probability 0, but 0 times an Inf or NaN value is NaN in the
// matrix product.  Such a product is never finite, so queries whose sums came out
// not finite are computed again by prompt_row, which skips hidden keys; the loop
// itself checks nothing.  Every query that meets such a value pays a wavefront's walk
// over its keys: 4 x 1000 tokens, 16 heads of 64, NaN in all padding, 30 us -> 6.9 ms.

// Wavefronts per SIMD: as many as the registers leave room for (two at every head size:
// 4x2048x32 heads of 64, causal, 116 us; three 98).
constexpr int prompt_waves(int hd) { return hd == 128 ? 2 : hd == 64 ? 3 : 4; }

template <typename T, int HD, bool CAP, bool BIAS, bool SPARSE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(prompt_waves(HD), prompt_waves(HD))))
void k_prompt_flash(gm_prompt_attention a) {
  constexpr int QB = 128, KB = 64, NW = 4;
  typedef typename Mfma32A<T>::vec vec;
  constexpr int KS = HD / 16;                 // k steps of S^T (head dim)
  constexpr int CB = HD / 32;                 // 32-channel blocks of O^T
  constexpr int CPR = HD / 8;                 // 16-byte chunks per key row
  constexpr int RPL = 16 / CPR;               // key rows per 256 bytes
  constexpr int RPI = 64 / CPR;               // key rows per 1 KB copy instruction
  constexpr int LPW = KB / RPI / NW;          // copy instructions per wavefront, tile and operand
  constexpr int TILE = KB * HD;
  __shared__ __attribute__((aligned(1024))) T sK0[TILE];
  __shared__ __attribute__((aligned(1024))) T sK1[TILE];
  __shared__ __attribute__((aligned(1024))) T sV0[TILE];
  __shared__ __attribute__((aligned(1024))) T sV1[TILE];
  __shared__ __attribute__((aligned(16))) int sDoc[2][KB];
  __shared__ unsigned long long sBits[2];     // key not masked (bit per key)
  __shared__ uint32_t sTiles[kTiles / 32];    // marks: some key of the tile may be visible
  __shared__ uint32_t sWhole[kTiles / 32];    // no key of it is masked, and all are of one document,
  __shared__ int sDocOf[kTiles];              // this one

  // query blocks outermost, heaviest first; the heads of a group next to one
  // another in steps of 8 workgroups where the key heads allow (one XCD, one L2)
  const int nqb = (a.Sq + QB - 1) / QB, P = a.B * a.n_heads;
  int p = blockIdx.x;
  {
    constexpr int kSlot = 256;
    const int sl = p / kSlot;
    if ((sl & 1) && (sl + 1) * kSlot <= nqb * P) p = sl * kSlot + (kSlot - 1 - (p - sl * kSlot));
  }
  const int blk = p / P, pair = p - blk * P;
  const int qb = a.causal ? nqb - 1 - blk : blk;
  const int b = pair / a.n_heads, hp = pair - b * a.n_heads;
  const int group = a.n_heads / a.kv_heads;
  const int kvh = hp % a.kv_heads, h = kvh * group + hp / a.kv_heads;
  const int Sq = a.Sq, S = a.Sk, off = a.q_offset;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int l32 = lane & 31, h2 = lane >> 5;
  const T* kbase = static_cast<const T*>(a.k.p) + b * a.k.batch + kvh * a.k.head;
  const T* vbase = static_cast<const T*>(a.v.p) + b * a.v.batch + kvh * a.v.head;
  const long long kld = a.k.token, vld = a.v.token;
  const int32_t* mk = SPARSE && a.key_mask ? a.key_mask + static_cast<long long>(b) * S : nullptr;
  const int32_t* kd = SPARSE && a.q_doc ? a.k_doc + static_cast<long long>(b) * S : nullptr;
  const int qw0 = qb * QB + wave * 32;        // first query of this wavefront
  const int qi = qw0 + l32;                   // this lane's query
  const int qpos = qi + off;
  const int pre = a.causal && a.prefix ? a.prefix[b] : 0;
  const bool causal = a.causal;

  vec qf[KS];
  {
    const int qc = qi < Sq ? qi : Sq - 1;
    const T* qp = static_cast<const T*>(a.q.p) + b * a.q.batch + qc * a.q.token + h * a.q.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const vec*>(qp + 16 * ks + 8 * h2);
  }
  int kend = S;
  if (causal) {
    const int last = (qb + 1) * QB + off;
    kend = last > pre ? last : pre;
    kend = kend < S ? kend : S;
  }
  const float c2 = CAP ? a.scores.scale * (2.f * kLog2e) / a.scores.softcap : a.scores.scale * kLog2e;
  const float capc = a.scores.softcap * kLog2e;
  const float slope2 = BIAS ? a.scores.slopes[h] * -kLog2e : 0.f;
  constexpr bool LOG2 = CAP || BIAS;          // scores are in log2 units before their maximum is taken

  const int qd = kd ? a.q_doc[static_cast<long long>(b) * Sq + (qi < Sq ? qi : Sq - 1)] : 0;
  if constexpr (SPARSE) {
    // 1024 keys a step, 4 keys a thread, up to 4 steps of loads in flight.  The last
    // threads read the row's last 4 keys, perhaps of the tile before: that tile's marks are
    // its own, and a mark too many on a tile not whole only has it looked at.
    constexpr int U = 4, STEP = 4 * 256;
    const int top = kend < kTiles * KB ? kend : kTiles * KB, own = 4 * static_cast<int>(threadIdx.x);
    i32x4 m[U], d[U];
    auto fetch = [&](int k0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        m[u] = i32x4{1, 1, 1, 1};
        d[u] = i32x4{0, 0, 0, 0};
        if (k0 + u * STEP >= top) break;
        const int key = k0 + u * STEP + own < S - 4 ? k0 + u * STEP + own : S - 4;
        if (mk) m[u] = *reinterpret_cast<const i32x4*>(mk + key);
        if (kd) d[u] = *reinterpret_cast<const i32x4*>(kd + key);
      }
    };
    if (S >= 4) fetch(0);
    int dmin = 0, dmax = 0;
    if (kd) {
      const int32_t* qds = a.q_doc + static_cast<long long>(b) * Sq;
      const int i0 = qb * QB + lane, i1 = i0 + 64;
      const int d0 = qds[i0 < Sq ? i0 : Sq - 1], d1 = qds[i1 < Sq ? i1 : Sq - 1];
      dmin = d0 < d1 ? d0 : d1;
      dmax = d0 < d1 ? d1 : d0;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const int x = __shfl_xor(dmin, o, 64), y = __shfl_xor(dmax, o, 64);
        dmin = x < dmin ? x : dmin;
        dmax = y > dmax ? y : dmax;
      }
    }
    // (fewer than 4 keys: one tile, looked at key by key)
    for (int i = threadIdx.x; i < kTiles / 32; i += 256) {
      sTiles[i] = S < 4;
      sWhole[i] = 0;
    }
    __syncthreads();
    for (int k0 = 0; k0 < top && S >= 4; k0 += U * STEP) {
      if (k0) fetch(k0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (k0 + u * STEP >= top) break;
        const int key = k0 + u * STEP + own;
        auto least = [](int x, int y) { return x < y ? x : y; };
        auto most = [](int x, int y) { return x < y ? y : x; };
        const int lo = least(least(d[u][0], d[u][1]), least(d[u][2], d[u][3]));
        const int hi = most(most(d[u][0], d[u][1]), most(d[u][2], d[u][3]));
        const int first = kd ? __shfl(lo, lane & 48, 64) : 0;   // of the tile's 16 lanes
        const bool any = key < S && (m[u][0] | m[u][1] | m[u][2] | m[u][3]) != 0 && lo <= dmax && hi >= dmin;
        const bool all = key + 4 <= S && m[u][0] != 0 && m[u][1] != 0 && m[u][2] != 0 && m[u][3] != 0 &&
                         lo == first && hi == first;
        const uint32_t on = static_cast<uint32_t>(__ballot(any) >> (lane & 48)) & 0xffffu;
        const uint32_t full = static_cast<uint32_t>(__ballot(all) >> (lane & 48)) & 0xffffu;
        const int t = key / KB;                  // (of the tile's first lane)
        if ((lane & 15) == 0 && on && t < kTiles) {
          atomicOr(&sTiles[t / 32], 1u << (t % 32));
          if (full == 0xffffu) atomicOr(&sWhole[t / 32], 1u << (t % 32));
          if (kd) sDocOf[t] = first;
        }
      }
    }
    __syncthreads();
  }
  // first key of the next tile to visit at or after t (a multiple of KB)
  auto next_tile = [&](int t) {
    if (!SPARSE) return t;
    while (t < kend && t < kTiles * KB) {
      const int i = t / KB;
      const uint32_t w = __builtin_amdgcn_readfirstlane(sTiles[i / 32]) >> (i % 32);
      if (w) return t + KB * __builtin_ctz(w);
      t = (i / 32 + 1) * 32 * KB;
    }
    return t;
  };
  // the tile at t, past the last key too, needs mask and documents key by key
  auto mixed = [&](int t) {
    if (!SPARSE) return false;
    if (t >= kTiles * KB) return true;
    return !(__builtin_amdgcn_readfirstlane(sWhole[t / KB / 32]) >> (t / KB % 32) & 1);
  };

  float mrun = -INFINITY, lrun = 0.f;
  f32x16 oacc[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[c][i] = 0.f;

  // swizzles: chunk c of key row r sits at chunk position c ^ f(r) (k_flash)
  const int cr = lane / CPR, cpos = lane % CPR;
  int mraw = 1, draw = 0;                     // wavefront 0: mask and document of key kb + lane of the tile in flight
  auto issue = [&](int kb, bool mix, T* dk, T* dv) {
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
      const int r = (wave * LPW + j) * RPI + cr;
      int key = kb + r;
      key = key < S ? key : S - 1;
      const int fk = (r / RPL) % CPR, fv = 4 * ((r / RPL) % (CPR / 4));
      dma16(kbase + key * kld + 8 * (cpos ^ fk), dk + (wave * LPW + j) * RPI * HD);
      dma16(vbase + key * vld + 8 * (cpos ^ fv), dv + (wave * LPW + j) * RPI * HD);
    }
    if (wave == 0 && mix) {
      const int key = kb + lane < S ? kb + lane : S - 1;
      if (mk) mraw = mk[key];
      if (kd) draw = kd[key];
    }
  };
  const int kswz = (l32 / RPL) % CPR;
  const int g = lane >> 4, e4 = (lane & 15) >> 2, q4 = lane & 3;
  const int vrow = 4 * (g >> 1) + e4;
  const int vswz4 = (vrow / RPL) % (CPR / 4);
  const int vsub = 2 * (g & 1) + (q4 >> 1);
  const int vin = 4 * (q4 & 1);
  uint32_t vaddr[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) vaddr[c] = 2 * (vrow * HD + 8 * (4 * (c ^ vswz4) + vsub) + vin);

  // one key tile from stage BUF (the other stage receives the tile at `next`); mix,
  // next_mix: whether they need mask and documents key by key
  auto tile = [&](auto BUF, int kb, bool mix, int next, bool next_mix) {
    constexpr int buf = decltype(BUF)::value;
    T* sk = buf ? sK1 : sK0;
    T* sv = buf ? sV1 : sV0;
    if (wave == 0 && mix) {
      const unsigned long long bits = __ballot(mraw != 0);
      if (kd) sDoc[buf][lane] = draw;
      if (lane == 0) sBits[buf] = bits;
    }
    wait_vmcnt0();                              // this wavefront's copies of the tile landed
    __syncthreads();
    if (next < kend) issue(next, next_mix, buf ? sK0 : sK1, buf ? sV0 : sV1);
    // every key of the tile past this wavefront's queries and the prefix
    if (causal && kb > qw0 + 31 + off && kb >= pre) return;
    unsigned long long bits = S - kb >= KB ? ~0ull : (1ull << (S - kb)) - 1;
    bool docs = kd != nullptr;
    if (mix) {
      bits &= sBits[buf];
    } else if (docs) {
      const bool seen = sDocOf[kb / KB] == qd;
      if (__ballot(seen) == 0) return;
      bits = seen ? bits : 0;
      docs = false;
    }
    // ---- S^T = K Q^T: two 32-key blocks
    f32x16 sacc[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 16; ++i) sacc[kk][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const vec kf = *reinterpret_cast<const vec*>(sk + (32 * kk + l32) * HD + 8 * ((2 * ks + h2) ^ kswz));
        sacc[kk] = Mfma32A<T>::run(kf, qf[ks], sacc[kk]);
      }
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
          sacc[kk][i] = fmaf(slope2, fabsf(dist - static_cast<float>(32 * kk + 8 * (i >> 2) + (i & 3))),
                             CAP ? sacc[kk][i] : sacc[kk][i] * c2);
    }
    // ---- masks
    const int last = qw0 + off > pre - 1 ? qw0 + off : pre - 1;
    if (__ballot(bits != ~0ull) || docs || (causal && kb + KB - 1 > last)) {
      unsigned long long vis = bits;
      if (causal) {
        // keys up to the query's own position or before the prefix
        const int n = (qpos + 1 > pre ? qpos + 1 : pre) - kb;
        vis &= n >= KB ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1;
      }
      vis >>= 4 * h2;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          i32x4 kdoc;
          if (docs) kdoc = *reinterpret_cast<const i32x4*>(&sDoc[buf][32 * kk + 8 * i4 + 4 * h2]);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            bool ok = (vis >> (32 * kk + 8 * i4 + r)) & 1ull;
            if (docs) ok = ok && kdoc[r] == qd;
            sacc[kk][4 * i4 + r] = ok ? sacc[kk][4 * i4 + r] : -INFINITY;
          }
        }
    }
    // fp16 probabilities times 2^7 (at most 2^15): fewer fall below its smallest normal
    constexpr float kUp = std::is_same<T, f16_t>::value ? 7.f : 0.f;
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
      for (int c = 0; c < CB; ++c) oacc[c] *= alpha;
      mrun = mnew;
    }
    const float msub = mrun == -INFINITY ? 0.f : mrun - kUp;
    // ---- probabilities, their sum, and P^T as 16-bit B operands
    vec pb[4];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        u32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s0 = sacc[kk][8 * hf + 2 * j], s1 = sacc[kk][8 * hf + 2 * j + 1];
          const float p0 = __builtin_amdgcn_exp2f(LOG2 ? s0 - msub : fmaf(s0, c2, -msub));
          const float p1 = __builtin_amdgcn_exp2f(LOG2 ? s1 - msub : fmaf(s1, c2, -msub));
          lrun += p0 + p1;
          w[j] = pack2<T>(p0, p1);
        }
        pb[2 * kk + hf] = __builtin_bit_cast(vec, w);
      }
    }
    // ---- O^T += V^T P^T: four 16-key steps; the V^T operands of step
    // k2 + 1 are read while step k2 multiplies
    const uint32_t vb = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_vptr)sv));
    u32x2 vf[2][CB][2];
    auto vread = [&](auto K2, u32x2 (&dst)[CB][2]) {
      constexpr int k2 = decltype(K2)::value;
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        dst[c][0] = lds_read_tr16<(16 * k2) * HD * 2>(vb + vaddr[c]);
        dst[c][1] = lds_read_tr16<(16 * k2 + 8) * HD * 2>(vb + vaddr[c]);
      }
    };
    auto vmul = [&](int k2, u32x2 (&src)[CB][2]) {
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        u32x4 w;
        w[0] = src[c][0][0]; w[1] = src[c][0][1]; w[2] = src[c][1][0]; w[3] = src[c][1][1];
        oacc[c] = Mfma32A<T>::run(__builtin_bit_cast(vec, w), pb[k2], oacc[c]);
      }
    };
    vread(std::integral_constant<int, 0>(), vf[0]);
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
  int kb = next_tile(0);
  if (kb < kend) {
    bool mix = mixed(kb);
    issue(kb, mix, sK0, sV0);
    while (true) {
      const int n1 = next_tile(kb + KB);
      const bool mix1 = n1 < kend && mixed(n1);
      tile(std::integral_constant<int, 0>(), kb, mix, n1, mix1);
      if (n1 >= kend) break;
      kb = next_tile(n1 + KB);
      mix = kb < kend && mixed(kb);
      tile(std::integral_constant<int, 1>(), n1, mix1, kb, mix);
      if (kb >= kend) break;
    }
  }
  // ---- normalise and store: lane holds channels 32c + 8i + 4(lane/32) + r of its query
  const float L = lrun + __shfl_xor(lrun, 32, 64);
  float odd = 0.f * L;
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) odd = fmaf(oacc[c][i], 0.f, odd);
  const unsigned long long odd_lanes = __ballot(odd != 0.f);   // (NaN != 0)
  uint32_t again = static_cast<uint32_t>(odd_lanes) | static_cast<uint32_t>(odd_lanes >> 32);
  if (qi < Sq && !(again >> l32 & 1)) {
    const float inv = L > 0.f ? 1.f / L : 0.f;
    T* out = static_cast<T*>(a.out.p) + b * a.out.batch + qi * a.out.token + h * a.out.head;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x2 r2;
        r2[0] = pack2<T>(oacc[c][4 * i] * inv, oacc[c][4 * i + 1] * inv);
        r2[1] = pack2<T>(oacc[c][4 * i + 2] * inv, oacc[c][4 * i + 3] * inv);
        *reinterpret_cast<u32x2*>(out + 32 * c + 8 * i + 4 * h2) = r2;
      }
  }
  for (; __builtin_expect(again != 0, 0); again &= again - 1) {
    const int i = qw0 + __builtin_ctz(again);
    if (i < Sq) prompt_row<T, HD>(a, b, h, i);
  }
}

template <typename T, int HD>
void prompt_flash(const gm_prompt_attention& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((a.Sq + 127) / 128) * a.n_heads * a.B), block(256);
  const bool cap = a.scores.softcap > 0.f, bias = a.scores.slopes;
  const std::true_type yes;
  const std::false_type no;
  auto launch = [&](auto c, auto b) {
    auto go = [&](auto sparse) {
      hipLaunchKernelGGL((k_prompt_flash<T, HD, decltype(c)::value, decltype(b)::value, decltype(sparse)::value>),
                         grid, block, 0, s, a);
    };
    if (a.key_mask || a.q_doc) go(yes);
    else go(no);
  };
  if (cap && bias) launch(yes, yes);
  else if (cap) launch(yes, no);
  else if (bias) launch(no, yes);
  else launch(no, no);
}

}  // namespace

void launch_attention_prompt(const gm_prompt_attention& a, hipStream_t s) {
  auto head = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    if (a.dtype == kF32) prompt_f32<HD>(a, s);
    else if (a.dtype == kBF16) prompt_flash<bf16_t, HD>(a, s);
    else prompt_flash<f16_t, HD>(a, s);
  };
  if (a.head_dim == 32) head(std::integral_constant<int, 32>());
  else if (a.head_dim == 64) head(std::integral_constant<int, 64>());
  else head(std::integral_constant<int, 128>());
}

}  // namespace gm
