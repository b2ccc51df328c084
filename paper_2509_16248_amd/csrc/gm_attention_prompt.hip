// gm_attention_prompt.hip -- attention over whole prompts with modified scores
// (gm.h, gm_attention): a tanh cap, a bias by distance, and key, document and
// prefix masks next to the causal one; query heads may share key heads.
#include <math.h>

#include "gm_device.h"
#include "gm_ops.h"

namespace gm {

namespace {

// One query by one wavefront, a key per lane: two passes over the keys, the
// largest score, then the sums.  A key of weight 0 is skipped, so that nothing a
// hidden value holds can reach the sums.
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
    for (int c = 0; c < HD; ++c) s = fmaf(to_f32(q[c]), to_f32(k[c]), s);
    return modify_score(s * a.scores.scale, a.scores.softcap, slope, fabsf(static_cast<float>(qpos - j)));
  };
  float m = -INFINITY;
  for (int j0 = 0; j0 < kend; j0 += 64)
    if (visible(j0 + lane)) m = fmaxf(m, score(j0 + lane));
  m = wave_max(m);
  float l = 0.f, o[CL] = {};
  for (int j0 = 0; j0 < kend; j0 += 64) {
    const bool ok = visible(j0 + lane);
    float p = 0.f;
    if (ok) {
      const float s = score(j0 + lane);
      p = s == -INFINITY ? 0.f : expf(s - m);
    }
    l += p;
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
  l = wave_sum(l);
  T* out = static_cast<T*>(a.out.p) + b * a.out.batch + i * a.out.token + h * a.out.head;
#pragma unroll
  for (int c = 0; c < CL; ++c)
    if (lane + 64 * c < HD) out[lane + 64 * c] = from_f32<T>(l == 0.f ? 0.f : o[c] / l);
}

// A wavefront per (query, head).
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_prompt_rows(gm_prompt_attention a) {
  const uint64_t e = blockIdx.x * 4ull + (threadIdx.x >> 6);
  const int i = static_cast<int>(e % a.Sq);
  const uint64_t r = e / a.Sq;
  const int h = static_cast<int>(r % a.n_heads);
  if (r / a.n_heads >= static_cast<uint64_t>(a.B)) return;
  prompt_row<T, HD>(a, static_cast<int>(r / a.n_heads), h, i);
}

template <typename T>
void prompt_rows(const gm_prompt_attention& a, hipStream_t s) {
  const uint64_t rows = static_cast<uint64_t>(a.B) * a.Sq * a.n_heads;
  const dim3 grid(static_cast<unsigned>((rows + 3) / 4)), block(256);
  if (a.head_dim == 32) hipLaunchKernelGGL((k_prompt_rows<T, 32>), grid, block, 0, s, a);
  else if (a.head_dim == 64) hipLaunchKernelGGL((k_prompt_rows<T, 64>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_prompt_rows<T, 128>), grid, block, 0, s, a);
}

}  // namespace

void launch_attention_prompt(const gm_prompt_attention& a, hipStream_t s) {
  if (a.dtype == kF32) prompt_rows<float>(a, s);
  else if (a.dtype == kBF16) prompt_rows<bf16_t>(a, s);
  else prompt_rows<f16_t>(a, s);
}

}  // namespace gm
