// gm_kvq.hip -- a KV cache held in 8 or 4 bits: rows quantised as they are
// stored, read back, and attention of new tokens over the cache.  The layout
// and the arithmetic of a group are gm.h's (gm_kv_cache).
#include <math.h>

#include <type_traits>

#include "gm_device.h"
#include "gm_ops.h"

namespace gm {

namespace {

// 8 channels of a row in storage type T: 16 bytes, or two times 16 in fp32.
template <typename T> struct Row8 {
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

// float -> bfloat16 bits, round to nearest even (finite x), in integers: the
// scale of a group of subnormals is a subnormal too.
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

// Larger of v in the 4 lanes of a quad, in each of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  uint32_t w = __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
  v = v > w ? v : w;
  w = __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);            // lanes 2 3 0 1
  return v > w ? v : w;
}

// x / s rounded to the nearest integer, ties to even, limited to [-Q, Q].  The
// quotient by the hardware reciprocal is off by one at most; x - q s is exact
// in fp32 (s has 8 significant bits, q 7, and the difference is no larger than
// s / 2 or so), so comparing it with s / 2 settles the nearest integer.
template <int Q>
__device__ __forceinline__ int quantise(float x, float s, float inv) {
  float q = rintf(x * inv);
  const float r = fmaf(-q, s, x), half = 0.5f * s;
  const float a = fabsf(r);
  const bool odd = static_cast<int>(q) & 1;
  if (a > half || (a == half && odd)) q += r > 0.f ? 1.f : -1.f;
  return static_cast<int>(fminf(fmaxf(q, -static_cast<float>(Q)), static_cast<float>(Q)));
}

struct KvRows {
  gm_kv_cache c;
  gm_tensor k, v;
  const int32_t *start, *count, *mask;
  int B, n;
};

// Which row and channels a thread handles: 8 channels `ch` of head h of row i of
// sequence b, of k or v.  Channels run fastest, then the rows of a head, whose
// codes are contiguous in the cache.
struct KvPlace {
  int b, i, h, which, ch, pos;
  bool live;      // row within its count and position within the cache
};
template <int HD>
__device__ __forceinline__ bool kv_place(const KvRows& a, KvPlace& p) {
  constexpr int C8 = HD / 8;
  const uint64_t e = blockIdx.x * 256ull + threadIdx.x;
  p.ch = static_cast<int>(e % C8) * 8;
  uint64_t r = e / C8;
  p.i = static_cast<int>(r % a.n);
  r /= a.n;
  p.which = static_cast<int>(r & 1);
  r >>= 1;
  p.h = static_cast<int>(r % a.c.heads);
  r /= a.c.heads;
  if (r >= static_cast<uint64_t>(a.B)) return false;
  p.b = static_cast<int>(r);
  const long long pos = static_cast<long long>(a.start ? a.start[p.b] : 0) + p.i;
  p.live = pos >= 0 && pos < a.c.max_seq && (!a.count || p.i < a.count[p.b]);
  p.pos = p.live ? static_cast<int>(pos) : 0;
  return true;
}

// One thread per 8 channels of a row, 4 threads (a quad of lanes) per group.
// The threads of a quad take the same branches: they share their row.
template <typename T, int HD, int BITS>
__global__ __launch_bounds__(256) void k_kv_write(KvRows a) {
  constexpr int Q = BITS == 8 ? 127 : 7, OFF = 1 << (BITS - 1);
  KvPlace p;
  if (!kv_place<HD>(a, p) || !p.live) return;
  const gm_tensor& src = p.which ? a.v : a.k;
  Row8<T> row;
  row.load(static_cast<const T*>(src.p) + p.b * src.batch + p.i * src.token + p.h * src.head + p.ch);
  float x[8];
  uint32_t amax = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = row.get(j);
    const uint32_t u = __float_as_uint(x[j]) & 0x7fffffffu;
    amax = u > amax ? u : amax;
  }
  amax = quad_max(amax);
  const bool finite = amax < 0x7f800000u;
  const uint32_t sb = finite ? bf16_bits(__uint_as_float(amax) * (1.0f / Q)) : 0x7fc0u;
  // a scale whose reciprocal would overflow, or whose half be inexact: both
  // sides of the quotient times 2^64 (exact)
  const float up = amax < (40u << 23) ? 18446744073709551616.f : 1.f;
  const float s = bf16_value(sb) * up;
  const bool zero = !finite || s == 0.f;
  const float inv = zero ? 0.f : __builtin_amdgcn_rcpf(s);
  uint32_t code[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    code[j] = static_cast<uint32_t>((zero ? 0 : quantise<Q>(x[j] * up, s, inv)) + OFF);
  const long long head = static_cast<long long>(p.b) * a.c.heads + p.h;
  char* codes = static_cast<char*>(p.which ? a.c.v : a.c.k) +
                (head * a.c.max_seq + p.pos) * (HD * BITS / 8) + p.ch * BITS / 8;
  if constexpr (BITS == 8) {
    u32x2 w;
    w[0] = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
    w[1] = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
    *reinterpret_cast<u32x2*>(codes) = w;
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w |= code[j] << (4 * j);
    *reinterpret_cast<uint32_t*>(codes) = w;
  }
  if (p.ch % kKvGroup == 0) {
    uint16_t* sc = static_cast<uint16_t*>(p.which ? a.c.v_scale : a.c.k_scale);
    sc[(head * (HD / kKvGroup) + p.ch / kKvGroup) * a.c.max_seq + p.pos] = static_cast<uint16_t>(sb);
  }
  if (a.c.valid && p.h == 0 && p.which == 0 && p.ch == 0)
    a.c.valid[static_cast<long long>(p.b) * a.c.max_seq + p.pos] =
        !a.mask || a.mask[static_cast<long long>(p.b) * a.n + p.i] != 0;
}

template <typename T, int HD, int BITS>
__global__ __launch_bounds__(256) void k_kv_read(KvRows a) {
  constexpr int OFF = 1 << (BITS - 1);
  KvPlace p;
  if (!kv_place<HD>(a, p)) return;
  Row8<T> row;
  if (p.live) {
    const long long head = static_cast<long long>(p.b) * a.c.heads + p.h;
    const char* codes = static_cast<const char*>(p.which ? a.c.v : a.c.k) +
                        (head * a.c.max_seq + p.pos) * (HD * BITS / 8) + p.ch * BITS / 8;
    const uint16_t* sc = static_cast<const uint16_t*>(p.which ? a.c.v_scale : a.c.k_scale);
    const float s = bf16_value(sc[(head * (HD / kKvGroup) + p.ch / kKvGroup) * a.c.max_seq + p.pos]);
    if constexpr (BITS == 8) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(codes);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        row.set(j, static_cast<float>(static_cast<int>((w[j / 4] >> (8 * (j % 4))) & 255u) - OFF) * s);
    } else {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(codes);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        row.set(j, static_cast<float>(static_cast<int>((w >> (4 * j)) & 15u) - OFF) * s);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) row.set(j, 0.f);
  }
  const gm_tensor& dst = p.which ? a.v : a.k;
  row.store(static_cast<T*>(dst.p) + p.b * dst.batch + p.i * dst.token + p.h * dst.head + p.ch);
}

// f(storage type, head size, bits) with the three as compile-time values.
template <typename F>
void by_cache(int dtype, const gm_kv_cache& c, F f) {
  auto bits = [&](auto t, auto hd) {
    if (c.bits == 8) f(t, hd, std::integral_constant<int, 8>());
    else f(t, hd, std::integral_constant<int, 4>());
  };
  auto head = [&](auto t) {
    if (c.head_dim == 32) bits(t, std::integral_constant<int, 32>());
    else if (c.head_dim == 64) bits(t, std::integral_constant<int, 64>());
    else bits(t, std::integral_constant<int, 128>());
  };
  if (dtype == kF32) head(float());
  else if (dtype == kBF16) head(bf16_t());
  else head(f16_t());
}

uint32_t kv_blocks(const KvRows& a) {
  return static_cast<uint32_t>(
      (static_cast<uint64_t>(a.B) * a.n * a.c.heads * 2 * (a.c.head_dim / 8) + 255) / 256);
}

}  // namespace

void launch_kv_write(const gm_kv_cache& c, int dtype, int B, int n, const gm_tensor& k,
                     const gm_tensor& v, const int32_t* start, const int32_t* count,
                     const int32_t* mask, hipStream_t s) {
  const KvRows a{c, k, v, start, count, mask, B, n};
  by_cache(dtype, c, [&](auto t, auto hd, auto bits) {
    hipLaunchKernelGGL((k_kv_write<decltype(t), decltype(hd)::value, decltype(bits)::value>),
                       dim3(kv_blocks(a)), dim3(256), 0, s, a);
  });
}

void launch_kv_read(const gm_kv_cache& c, int dtype, int B, int n, const int32_t* start,
                    const int32_t* count, const gm_tensor& k, const gm_tensor& v, hipStream_t s) {
  const KvRows a{c, k, v, start, count, nullptr, B, n};
  by_cache(dtype, c, [&](auto t, auto hd, auto bits) {
    hipLaunchKernelGGL((k_kv_read<decltype(t), decltype(hd)::value, decltype(bits)::value>),
                       dim3(kv_blocks(a)), dim3(256), 0, s, a);
  });
}

// ------------------------------------------------------------ attention over the cache
namespace {

// Key chunks per sequence and key head: chunk s of sequence b covers keys
// [s, s + 1) * ceil(length / nsplit), rounded up to whole tiles of 64.
int cached_splits(const gm_kv_cache& c, int B, int Sq, int n_heads) {
  const long long rows = static_cast<long long>(B) * Sq * n_heads;
  long long want = (1024 + rows - 1) / rows;
  const long long most = (c.max_seq + 255) / 256;
  want = want < most ? want : most;
  return static_cast<int>(want < 64 ? want : 64);
}

// Workgroup = one query row (sequence, token, head) and one chunk of its keys.
// HD / 8 lanes hold a key row, 8 channels each; every lane group keeps an
// online softmax of its own, merged by shuffles and in LDS.  With one chunk the
// workgroup writes the output, else (m, l, o) to the workspace.
template <typename T, int HD, int BITS>
__global__ __launch_bounds__(256) void k_cached_rows(gm_cached_attention a, gm_kv_cache c,
                                                     int nsplit) {
  constexpr int OFF = 1 << (BITS - 1), NWV = 4;
  constexpr int G = HD / 8, KPW = 64 / G, NG = NWV * KPW;
  __shared__ float s_m[NWV], s_l[NWV], s_o[NWV][HD];
  const int row = blockIdx.x, split = blockIdx.y;
  const int h = row % a.n_heads, i = row / a.n_heads % a.Sq, b = row / a.n_heads / a.Sq;
  const int kvh = h / (a.n_heads / c.heads);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int grp = lane / G, gl = lane % G;
  int len = a.lengths[b];
  len = len < c.max_seq ? len : c.max_seq;
  const int qpos = len - a.Sq + i;
  const int per = len > 0 ? (len + 64 * nsplit - 1) / (64 * nsplit) * 64 : 0;
  const int k0 = split * per;
  int k1 = k0 + per;
  k1 = k1 < qpos + 1 ? k1 : qpos + 1;
  const float slope = a.scores.slopes ? a.scores.slopes[h] : 0.f;
  float q[8];
  {
    Row8<T> r;
    r.load(static_cast<const T*>(a.q.p) + b * a.q.batch + i * a.q.token + h * a.q.head + 8 * gl);
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = r.get(j);
  }
  const long long head = static_cast<long long>(b) * c.heads + kvh;
  const char* kc = static_cast<const char*>(c.k) + head * c.max_seq * (HD * BITS / 8) + gl * BITS;
  const char* vc = static_cast<const char*>(c.v) + head * c.max_seq * (HD * BITS / 8) + gl * BITS;
  const long long sbase = (head * (HD / kKvGroup) + gl / 4) * c.max_seq;
  const uint16_t* ks = static_cast<const uint16_t*>(c.k_scale) + sbase;
  const uint16_t* vs = static_cast<const uint16_t*>(c.v_scale) + sbase;
  const uint8_t* valid = c.valid ? c.valid + static_cast<long long>(b) * c.max_seq : nullptr;
  auto codes = [&](const char* p, float (&x)[8]) {
    if constexpr (BITS == 8) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = static_cast<float>(static_cast<int>((w[j / 4] >> (8 * (j % 4))) & 255u) - OFF);
    } else {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        x[j] = static_cast<float>(static_cast<int>((w >> (4 * j)) & 15u) - OFF);
    }
  };
  float m = -INFINITY, l = 0.f, o[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = 0.f;
  for (int key = k0 + wave * KPW + grp; key < k1; key += NG) {
    float kx[8], vx[8];
    codes(kc + static_cast<long long>(key) * (HD * BITS / 8), kx);
    codes(vc + static_cast<long long>(key) * (HD * BITS / 8), vx);
    const float sk = bf16_value(ks[key]), sv = bf16_value(vs[key]);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(q[j], kx[j], s);
    s *= sk;
#pragma unroll
    for (int off = G / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    if (valid && !valid[key]) continue;   // the same for the whole lane group
    s = modify_score(s * a.scores.scale, a.scores.softcap, slope, static_cast<float>(qpos - key));
    const float mn = fmaxf(m, s);
    const float corr = m == mn ? 1.f : expf(m - mn), p = s == -INFINITY ? 0.f : expf(s - mn);
    l = l * corr + p;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = o[j] * corr + p * sv * vx[j];
    m = mn;
  }
#pragma unroll
  for (int off = G; off < 64; off <<= 1) {
    const float mo = __shfl_xor(m, off, 64), lo = __shfl_xor(l, off, 64);
    const float mm = fmaxf(m, mo);
    const float w0 = m == -INFINITY ? 0.f : expf(m - mm);
    const float w1 = mo == -INFINITY ? 0.f : expf(mo - mm);
    l = l * w0 + lo * w1;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = o[j] * w0 + __shfl_xor(o[j], off, 64) * w1;
    m = mm;
  }
  if (lane < G) {
    if (lane == 0) {
      s_m[wave] = m;
      s_l[wave] = l;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s_o[wave][8 * gl + j] = o[j];
  }
  __syncthreads();
  const int ch = threadIdx.x;
  if (ch >= HD) return;
  float M = -INFINITY, L = 0.f, O = 0.f;
  for (int w = 0; w < NWV; ++w) M = fmaxf(M, s_m[w]);
  for (int w = 0; w < NWV; ++w) {
    const float f = s_m[w] == -INFINITY ? 0.f : expf(s_m[w] - M);
    L += s_l[w] * f;
    O += s_o[w][ch] * f;
  }
  if (nsplit == 1) {
    T* out = static_cast<T*>(a.out.p) + b * a.out.batch + i * a.out.token + h * a.out.head;
    out[ch] = from_f32<T>(L == 0.f ? 0.f : O / L);
    return;
  }
  float* part = static_cast<float*>(a.workspace) +
                (static_cast<long long>(row) * nsplit + split) * (HD + 2);
  part[2 + ch] = O;
  if (ch == 0) {
    part[0] = M;
    part[1] = L;
  }
}

// The chunks of a row merged in their order.
template <typename T, int HD>
__global__ __launch_bounds__(HD) void k_cached_merge(gm_cached_attention a, int nsplit) {
  const int row = blockIdx.x, ch = threadIdx.x;
  const int h = row % a.n_heads, i = row / a.n_heads % a.Sq, b = row / a.n_heads / a.Sq;
  const float* part = static_cast<const float*>(a.workspace) +
                      static_cast<long long>(row) * nsplit * (HD + 2);
  float M = -INFINITY, L = 0.f, O = 0.f;
  for (int s = 0; s < nsplit; ++s) M = fmaxf(M, part[s * (HD + 2)]);
  for (int s = 0; s < nsplit; ++s) {
    const float ms = part[s * (HD + 2)];
    const float f = ms == -INFINITY ? 0.f : expf(ms - M);
    L += part[s * (HD + 2) + 1] * f;
    O += part[s * (HD + 2) + 2 + ch] * f;
  }
  T* out = static_cast<T*>(a.out.p) + b * a.out.batch + i * a.out.token + h * a.out.head;
  out[ch] = from_f32<T>(L == 0.f ? 0.f : O / L);
}

}  // namespace

uint64_t attention_cached_workspace(const gm_kv_cache& c, int, int B, int Sq, int n_heads) {
  if (B == 0 || Sq == 0) return 0;
  const int nsplit = cached_splits(c, B, Sq, n_heads);
  if (nsplit == 1) return 0;
  return static_cast<uint64_t>(B) * Sq * n_heads * nsplit * (c.head_dim + 2) * sizeof(float);
}

void launch_attention_cached(const gm_cached_attention& a, hipStream_t s) {
  const gm_kv_cache& c = *a.cache;
  const int nsplit = cached_splits(c, a.B, a.Sq, a.n_heads);
  const unsigned rows = static_cast<unsigned>(a.B) * a.Sq * a.n_heads;
  by_cache(a.dtype, c, [&](auto t, auto hd, auto bits) {
    typedef decltype(t) T;
    constexpr int HD = decltype(hd)::value;
    hipLaunchKernelGGL((k_cached_rows<T, HD, decltype(bits)::value>), dim3(rows, nsplit), dim3(256),
                       0, s, a, c, nsplit);
    if (nsplit > 1)
      hipLaunchKernelGGL((k_cached_merge<T, HD>), dim3(rows), dim3(HD), 0, s, a, nsplit);
  });
}

}  // namespace gm
