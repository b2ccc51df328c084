// gm_flash.h -- what the MFMA attention kernels share: the 32x32x16 matrix
// instruction by storage type, 16-bit packing, copies into LDS and transposing
// reads of it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gm_device.h"

namespace gm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T> struct Mfma32A;
template <> struct Mfma32A<bf16_t> {
  typedef bf16x8 vec;
  static __device__ __forceinline__ f32x16 run(vec a, vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma32A<f16_t> {
  typedef f16x8 vec;
  static __device__ __forceinline__ f32x16 run(vec a, vec b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

constexpr float kTau = 8.0f;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));

// Two floats rounded to T (nearest even) in one 32-bit word, lo first: one
// v_cvt_pk_bf16_f32 for bf16.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<bf16_t>(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2v));
}
template <> __device__ __forceinline__ uint32_t pack2<f16_t>(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2v));
}

typedef __attribute__((address_space(3))) void* lds_vptr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16 bytes from global memory straight into LDS (global_load_lds_dwordx4):
// lane i of the wavefront writes bytes [16i, 16i + 16) from `lds`, which
// must be the same for every lane.
__device__ __forceinline__ void dma16(const void* g, void* lds) {
  __builtin_amdgcn_global_load_lds(g, (lds_vptr)lds, 16, 0, 0);
}

// ds_read_b64_tr_b16: in each group of 16 lanes, lane i receives element
// (i % 4) of the 4-element rows read by lanes i/4, 4 + i/4, 8 + i/4 and
// 12 + i/4 of its group, in that order.  Issued as inline assembly: the
// compiler would otherwise make this read wait for every LDS copy in
// flight (it cannot tell that they fill the other stage).  Its result is
// therefore invisible to the compiler's wait counting; lgkm_wait() below
// must precede any use.
template <int OFF>
__device__ __forceinline__ u32x2 lds_read_tr16(uint32_t addr) {
  u32x2 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF) : "memory");
  return v;
}

// Wait until at most N LDS reads are outstanding (LDS reads complete in
// issue order; no scalar memory read is in flight here), then tie the
// values to the wait so that no use moves above it.
template <int N>
__device__ __forceinline__ void lgkm_wait(u32x2* v, int n) {
  static_assert(N >= 0 && N < 16, "lgkmcnt range");
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"i"(N) : "memory");
  for (int i = 0; i < n; ++i) asm volatile("" : "+v"(v[i]));
}

__device__ __forceinline__ void wait_vmcnt0() {
  __builtin_amdgcn_s_waitcnt((0x7 << 4) | (0xF << 8));   // vmcnt(0), others untouched
}

}  // namespace gm
