// gm_ops.h -- launch functions of the operators on caller tensors (gm.h,
// "operators"), and the score arithmetic they share.  The arguments have been
// checked; every function only enqueues.
#pragma once
#include <math.h>

#include "gm.h"
#include "gm_device.h"
#include "gm_kernels.h"

namespace gm {

constexpr int kKvGroup = 32;   // channels per scale of a quantised cache

// Caps of scores.  The 16-bit kernels take softcap tanh(x) as softcap - 2 softcap /
// (exp(2 x) + 1), off by 2^-23 softcap or so whatever x is: 1.2e-4 at the largest.
constexpr float kLeastCap = 1e-6f, kLargestCap = 1024.f;

void launch_kv_write(const gm_kv_cache& c, int dtype, int B, int n, const gm_tensor& k,
                     const gm_tensor& v, const int32_t* start, const int32_t* count,
                     const int32_t* mask, hipStream_t s);
void launch_kv_read(const gm_kv_cache& c, int dtype, int B, int n, const int32_t* start,
                    const int32_t* count, const gm_tensor& k, const gm_tensor& v, hipStream_t s);
void launch_attention_cached(const gm_cached_attention& a, hipStream_t s);
uint64_t attention_cached_workspace(const gm_kv_cache& c, int dtype, int B, int Sq, int n_heads);
void launch_attention_prompt(const gm_prompt_attention& a, hipStream_t s);

// softcap * tanh(s / softcap) - slope * distance of a scaled score, in fp32.
__device__ __forceinline__ float modify_score(float s, float softcap, float slope, float distance) {
  if (softcap > 0.f) s = softcap * tanhf(s / softcap);
  return fmaf(-slope, distance, s);
}

}  // namespace gm
