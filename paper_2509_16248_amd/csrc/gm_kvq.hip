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
  // Past the caches (1 x 2048 x 32 heads of 128, 4 bits, 10.5 us, plain stores 11.4; 2 x
  // 3000 x 8 heads 7.9 and 9.5).  An attention that reads the rows next has them from the
  // Infinity Cache either way: both calls together 56.2 and 55.9, 72.0 and 72.7.
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) __builtin_nontemporal_store(raw[i], reinterpret_cast<u32x4*>(p) + i);
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

// 8 channels' bits without their signs, the largest in each half of the word (16-bit
// types; Inf and NaN are the largest) or the largest (fp32).
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}
template <typename T>
__device__ __forceinline__ uint32_t largest_bits(const Row8<T>& row) {
  uint32_t m = 0;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = row.raw[i / 4][i % 4] & 0x7fffffffu;
      m = u > m ? u : m;
    }
    return quad_max(m);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max_u16x2(m, row.raw[0][i] & 0x7fff7fffu);
    m = m >> 16 > (m & 0xffffu) ? m >> 16 : m & 0xffffu;
    m = quad_max(m);
    return __float_as_uint(to_f32(__builtin_bit_cast(T, static_cast<uint16_t>(m))));
  }
}

// x / s rounded to the nearest integer (ties to even), limited to [-Q, Q], plus
// 2^(BITS - 1), in the low byte of the result (the bytes above are not 0).  The
// quotient is refined once, to 2^-45 of itself before it is rounded to fp32, and
// that settles the integer: a quotient on a half k + 1/2 is an fp32 number and
// comes out exact, and any other of a 24-bit x and an 8-bit s lies more than
// (1 + 2^-8) half steps of fp32 away from one.  Adding 1.5 2^23 rounds it.
template <int BITS>
__device__ __forceinline__ uint32_t quantise(float x, float s, float inv) {
  constexpr float Q = BITS == 8 ? 127.f : 7.f, kRound = 12582912.f + (1 << (BITS - 1));
  float q = x * inv;
  q = fmaf(fmaf(-q, s, x), inv, q);
  return __float_as_uint(__builtin_amdgcn_fmed3f(q, -Q, Q) + kRound);
}
// Bytes 0 of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u),
                               __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// x / d and x % d of 32-bit numbers by one multiplication: m = ceil(2^(32 + s) / d) less
// 2^32, 2^s >= d.
struct Div {
  uint32_t d, m, s;
  Div() : d(1), m(0), s(0) {}
  explicit Div(uint32_t divisor) : d(divisor), s(0) {
    while (s < 32 && (1ull << s) < d) ++s;
    m = static_cast<uint32_t>(((1ull << 32) * ((1ull << s) - d)) / d + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t x, uint32_t& rest) const {
    const uint32_t t = __umulhi(m, x);
    const uint32_t q = s ? (t + ((x - t) >> 1)) >> (s - 1) : x;
    rest = x - q * d;
    return q;
  }
};

struct KvRows {
  gm_kv_cache c;
  gm_tensor k, v;
  const int32_t *start, *count, *mask;
  int B, n;
  Div by_n, by_heads, by_blocks;
};

// Which row and channels an item is: 8 channels `ch` of head h of row i of
// sequence b, of k or v.  Channels run fastest, then the rows of a head, whose
// codes are contiguous in the cache.
struct KvPlace {
  int b, i, h, which, ch, pos;
  bool some;      // there is such a row
  bool live;      // row within its count and position within the cache
};
// Item u of a thread.  U = 1: items of every head in one line.  U > 1: a workgroup's
// 256 U items are of one head, so that all but row and channel is the same for all of
// its threads and stays in scalar registers.
template <int HD, int U>
__device__ __forceinline__ KvPlace kv_place(const KvRows& a, int u) {
  constexpr uint32_t C8 = HD / 8;
  KvPlace p;
  uint32_t i, h, r;
  if constexpr (U == 1) {
    const uint64_t e = blockIdx.x * 256ull + threadIdx.x;
    p.ch = static_cast<int>(e % C8) * 8;
    r = a.by_n.div(static_cast<uint32_t>(e / C8), i);   // (a launch has fewer than 2^32 items)
  } else {
    uint32_t blk;
    r = __builtin_amdgcn_readfirstlane(a.by_blocks.div(blockIdx.x, blk));
    const uint32_t e = (blk * U + u) * 256 + threadIdx.x;
    p.ch = static_cast<int>(e % C8) * 8;
    i = e / C8;
  }
  p.i = static_cast<int>(i);
  p.which = static_cast<int>(r & 1);
  uint32_t b = a.by_heads.div(r >> 1, h);
  if constexpr (U > 1) {
    b = __builtin_amdgcn_readfirstlane(b);
    h = __builtin_amdgcn_readfirstlane(h);
  }
  p.h = static_cast<int>(h);
  p.some = b < static_cast<uint32_t>(a.B) && i < static_cast<uint32_t>(a.n);
  p.b = b < static_cast<uint32_t>(a.B) ? static_cast<int>(b) : 0;
  const long long pos = static_cast<long long>(a.start ? a.start[p.b] : 0) + p.i;
  p.live = p.some && pos >= 0 && pos < a.c.max_seq && (!a.count || p.i < a.count[p.b]);
  p.pos = p.live ? static_cast<int>(pos) : 0;
  return p;
}
template <int HD, int BITS>
__device__ __forceinline__ char* kv_codes(const KvRows& a, const KvPlace& p) {
  const long long head = static_cast<long long>(p.b) * a.c.heads + p.h;
  return static_cast<char*>(p.which ? a.c.v : a.c.k) +
         (head * a.c.max_seq + p.pos) * (HD * BITS / 8) + p.ch * BITS / 8;
}
template <int HD>
__device__ __forceinline__ uint16_t* kv_scale(const KvRows& a, const KvPlace& p) {
  const long long head = static_cast<long long>(p.b) * a.c.heads + p.h;
  return static_cast<uint16_t*>(p.which ? a.c.v_scale : a.c.k_scale) +
         (head * (HD / kKvGroup) + p.ch / kKvGroup) * a.c.max_seq + p.pos;
}
template <typename T>
__device__ __forceinline__ T* kv_row(const KvRows& a, const KvPlace& p) {
  const gm_tensor& t = p.which ? a.v : a.k;
  return static_cast<T*>(t.p) + p.b * t.batch + p.i * t.token + p.h * t.head + p.ch;
}

// A thread takes U items of 8 channels, 256 apart, their loads up front; 4 threads
// (a quad of lanes) share a group, and with it their row and their branches.
template <typename T, int HD, int BITS, int U>
__global__ __launch_bounds__(256) void k_kv_write(KvRows a) {
  constexpr int Q = BITS == 8 ? 127 : 7;
  KvPlace place[U];
  Row8<T> rows[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    place[u] = kv_place<HD, U>(a, u);
    if (place[u].live) rows[u].load(kv_row<const T>(a, place[u]));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const KvPlace& p = place[u];
    if (!p.live) continue;
    const uint32_t amax = largest_bits(rows[u]);
    const bool finite = amax < 0x7f800000u;
    const uint32_t sb = finite ? bf16_bits(__uint_as_float(amax) * (1.0f / Q)) : 0x7fc0u;
    float x[8], s = bf16_value(sb);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = rows[u].get(j);
    if (__builtin_expect(amax < (40u << 23), 0)) {
      // a scale whose reciprocal would overflow: both sides of the quotient times 2^64
      s *= 18446744073709551616.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= 18446744073709551616.f;
    }
    const float inv = s == 0.f ? 0.f : __builtin_amdgcn_rcpf(s);
    uint32_t code[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) code[j] = quantise<BITS>(x[j], s, inv);
    char* codes = kv_codes<HD, BITS>(a, p);
    if constexpr (BITS == 8) {
      u32x2 w;
      w[0] = low_bytes(code[0], code[1], code[2], code[3]);
      w[1] = low_bytes(code[4], code[5], code[6], code[7]);
      *reinterpret_cast<u32x2*>(codes) = w;
    } else {
      *reinterpret_cast<uint32_t*>(codes) = low_bytes(code[0], code[2], code[4], code[6]) |
                                            low_bytes(code[1], code[3], code[5], code[7]) << 4;
    }
    if (p.ch % kKvGroup == 0) *kv_scale<HD>(a, p) = static_cast<uint16_t>(sb);
    if (a.c.valid && p.h == 0 && p.which == 0 && p.ch == 0)
      a.c.valid[static_cast<long long>(p.b) * a.c.max_seq + p.pos] =
          !a.mask || a.mask[static_cast<long long>(p.b) * a.n + p.i] != 0;
  }
}

template <typename T, int HD, int BITS, int U>
__global__ __launch_bounds__(256) void k_kv_read(KvRows a) {
  constexpr int OFF = 1 << (BITS - 1);
  KvPlace place[U];
  u32x2 w[U];
  uint16_t sb[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    place[u] = kv_place<HD, U>(a, u);
    w[u] = u32x2{0, 0};
    sb[u] = 0;
    if (place[u].live) {
      const char* codes = kv_codes<HD, BITS>(a, place[u]);
      if constexpr (BITS == 8) w[u] = *reinterpret_cast<const u32x2*>(codes);
      else w[u][0] = *reinterpret_cast<const uint32_t*>(codes);
      sb[u] = *kv_scale<HD>(a, place[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!place[u].some) continue;
    const float s = bf16_value(sb[u]);
    Row8<T> row;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = BITS == 8 ? (w[u][j / 4] >> (8 * (j % 4))) & 255u : (w[u][0] >> (4 * j)) & 15u;
      // (code - OFF) s, exact in fp32 up to its largest number (which OFF s by itself may
      // pass); rows that are not there have s = 0 and become +0
      row.set(j, fmaf(static_cast<float>(code) - OFF, s, 0.f));
    }
    row.store(kv_row<T>(a, place[u]));
  }
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

// f(items per thread, rows, grid): four items a thread where a head's rows fill such a
// workgroup, one where they do not.
template <typename F>
void kv_launch(KvRows a, F f) {
  const uint64_t heads = static_cast<uint64_t>(a.B) * a.c.heads * 2;
  const uint64_t items = static_cast<uint64_t>(a.n) * (a.c.head_dim / 8);   // of a head
  a.by_n = Div(a.n);
  a.by_heads = Div(a.c.heads);
  if (items >= 1024) {
    const uint64_t blocks = (items + 1023) / 1024;
    a.by_blocks = Div(static_cast<uint32_t>(blocks));
    f(std::integral_constant<int, 4>(), a, dim3(static_cast<uint32_t>(heads * blocks)));
  } else {
    f(std::integral_constant<int, 1>(), a, dim3(static_cast<uint32_t>((heads * items + 255) / 256)));
  }
}

}  // namespace

void launch_kv_write(const gm_kv_cache& c, int dtype, int B, int n, const gm_tensor& k,
                     const gm_tensor& v, const int32_t* start, const int32_t* count,
                     const int32_t* mask, hipStream_t s) {
  kv_launch(KvRows{c, k, v, start, count, mask, B, n}, [&](auto u, const KvRows& a, dim3 grid) {
    by_cache(dtype, c, [&](auto t, auto hd, auto bits) {
      hipLaunchKernelGGL((k_kv_write<decltype(t), decltype(hd)::value, decltype(bits)::value, decltype(u)::value>),
                         grid, dim3(256), 0, s, a);
    });
  });
}

void launch_kv_read(const gm_kv_cache& c, int dtype, int B, int n, const int32_t* start,
                    const int32_t* count, const gm_tensor& k, const gm_tensor& v, hipStream_t s) {
  kv_launch(KvRows{c, k, v, start, count, nullptr, B, n}, [&](auto u, const KvRows& a, dim3 grid) {
    by_cache(dtype, c, [&](auto t, auto hd, auto bits) {
      hipLaunchKernelGGL((k_kv_read<decltype(t), decltype(hd)::value, decltype(bits)::value, decltype(u)::value>),
                         grid, dim3(256), 0, s, a);
    });
  });
}

// ------------------------------------------------------------ attention over the cache
//
// The cache is read once per row block of queries by workgroups that take chunks of
// the keys; each leaves, per query row, its largest score m (log2 units), the sum l
// of its exp2(score - m) and its own normalised output o, and the chunks of a row
// are merged as sum(w o) / sum(w), w = l exp2(m - largest m), in their order.
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Row r of key head kvh of sequence b: token r / G, query head kvh * G + r % G.
struct CachedPlan {
  int rows;         // query rows of a key head: Sq * (n_heads / heads)
  int blocks;       // row blocks of a key head
  int nsplit;       // key chunks per row block
  int waves;        // wavefronts of a workgroup of the MFMA kernel
};

// The MFMA kernel takes 16-bit dtypes: 16 columns of a product are shared by query
// rows and 32-channel groups.  In fp32 a workgroup takes one row.  Chunks: as many as
// bring 512 workgroups, two a CU, of 128 keys at the least (us a call at 256 / 512 /
// 768 / 1024 workgroups: one sequence of 32000 keys, 32 heads of 128, 4 bits, 46.1 /
// 38.0 / 38.2 / 41.8; 32 of 8190 with 8 heads 85.8 / 68.9 / 73.4 / 73.8; 8 of 2000 with
// 8 heads, 8 bits, 16.6 / 15.9 / 20.0 / 20.0; at 128 / 256 / 512 keys: one of 4000 keys
// with 8 heads 11.8 / 12.0 / 14.4).  Up to 65536 / head_dim positions one chunk, which
// saves the merge's launch (one chunk / split: 8 sequences, 12 heads of 64, 8 bits,
// capacity 1024, length 300 6.7 / 8.3, 640 8.1 / 9.1, 1000 10.5 / 10.4; capacity 2048, 2000
// 16.1 / 11.0; one, 32 heads of 128, 4 bits, capacity 256 6.4 / 7.9, 512 8.0 / 7.9, 1024
// 12.0 / 8.6): a call knows the capacity, a cache in use is half full on average.  Above it,
// 8 wavefronts in the one chunk: 8 x 12 heads of 64, 8 bits, capacity 1280, half full / full
// 7.2 / 10.1 against 8.3 / 10.9 split, 1792 8.2 / 12.0 against 10.4 / 12.1; one, 32 heads of
// 64, 4 bits, 1280 6.7 / 9.2 against 7.7 / 8.2, 1792 7.6 / 11.1 against 7.9 / 8.2; 4, 32/8 heads
// of 128, 8 bits, 640 7.8 / 10.4 against 8.6 / 8.9, 1024 9.4 / 13.3 against 8.7 / 9.6.  The
// fp32 kernel, one row a workgroup, wants 1024 of them (8 sequences of 2000 keys, 32/8
// heads of 128, at 256 / 512 / 1024 / 2048: 60.6 / 43.2 / 37.6 / 38.7) and half the positions
// (one, 12 heads of 64, capacity 1024, length 300 7.6 / 7.3, 1000 15.7 / 7.5).
// One or two chunks of at most 256 row blocks, one a CU: a single chunk of 8 wavefronts
// in place of 4 each, so no merge (4 / 8 wavefronts: 8 sequences, 12 heads of 64, 8 bits,
// capacity 1024, length 300 6.4 / 6.0, 1000 10.0 / 8.9; 4, 32 heads of 32, 4 bits, 1500
// 11.9 / 9.9; 32 of 8190, 32/8 heads of 128, 4 bits, 70.0 / 66.8, of 2000, 8 bits, 35.2 /
// 30.7); a capacity of 256 gives 8 wavefronts a tile each and stays at 4 (one, 32 heads
// of 128, 4 bits, length 200 6.3 / 6.6).
CachedPlan cached_plan(const gm_kv_cache& c, int dtype, int B, int Sq, int n_heads) {
  CachedPlan p;
  p.rows = Sq * (n_heads / c.heads);
  const int per_block = dtype == kF32 ? 1 : 16 / (c.head_dim / kKvGroup);
  p.blocks = (p.rows + per_block - 1) / per_block;
  const long long wgs = static_cast<long long>(B) * c.heads * p.blocks;
  const int target = dtype == kF32 ? 1024 : 512, room = dtype == kF32 ? 32768 : 65536;
  long long want = (target + wgs - 1) / wgs;
  const long long most = static_cast<long long>(c.max_seq) * c.head_dim > room ? (c.max_seq + 127) / 128 : 1;
  want = want < most ? want : most;
  p.nsplit = static_cast<int>(want < 64 ? want : 64);
  p.waves = 4;
  if (dtype != kF32 && p.nsplit <= 2 && wgs <= 256 && c.max_seq > 256) {
    p.nsplit = 1;
    p.waves = 8;
  }
  return p;
}

// What a workgroup works on: sequence, key head, row block and its chunk of the
// keys [k0, k1) of a sequence of len keys, whole tiles of 64.
struct CachedPlace {
  int b, kvh, blk, split, len, k0, k1;
  __device__ __forceinline__ CachedPlace(const gm_cached_attention& a, const gm_kv_cache& c,
                                         const CachedPlan& p) {
    // (heads fastest: the row blocks of a head come to one XCD where the heads are a
    // multiple of 8, and share its L2: 4 sequences of 16000 keys, 32/2 heads of 128, 8 bits,
    // 29.8 us with the blocks side by side, 25.9 so)
    int x = blockIdx.x;
    const int heads = a.B * c.heads;
    blk = x / heads;
    x -= blk * heads;
    kvh = x % c.heads;
    b = x / c.heads;
    split = blockIdx.y;
    len = a.lengths[b];
    len = len < c.max_seq ? len : c.max_seq;
    len = len > 0 ? len : 0;
    const int per = (len + 64 * p.nsplit - 1) / (64 * p.nsplit) * 64;
    k0 = split * per;
    k1 = k0 + per < len ? k0 + per : len;
  }
};

template <typename T>
__device__ __forceinline__ T* cached_out(const gm_cached_attention& a, const gm_kv_cache& c, int b,
                                         int kvh, int r) {
  const int G = a.n_heads / c.heads;
  return static_cast<T*>(a.out.p) + b * a.out.batch + (r / G) * a.out.token +
         (kvh * G + r % G) * a.out.head;
}
// (m, l, o[HD]) of a chunk
template <int HD>
__device__ __forceinline__ float* cached_part(const gm_cached_attention& a, const gm_kv_cache& c,
                                              const CachedPlan& p, int b, int kvh, int r, int split) {
  const long long row = (static_cast<long long>(b) * c.heads + kvh) * p.rows + r;
  return static_cast<float*>(a.workspace) + (row * p.nsplit + split) * (HD + 2);
}

// 1 / x of a sum of weights (0, or 1 and more), 0 for 0: refined once, shorter than a division.
__device__ __forceinline__ float over_sum(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return x == 0.f ? 0.f : fmaf(fmaf(-x, r, 1.f), r, r);
}

// One query row by a workgroup.  HD / 8 lanes hold a key row, 8 channels each; every
// lane group keeps an online softmax of its own, merged by shuffles and in LDS.
template <typename T, int HD, int BITS>
__global__ __launch_bounds__(256) void k_cached_rows(gm_cached_attention a, gm_kv_cache c,
                                                     CachedPlan plan) {
  constexpr int OFF = 1 << (BITS - 1), NWV = 4;
  constexpr int G = HD / 8, KPW = 64 / G, NG = NWV * KPW;
  __shared__ float s_m[NWV], s_l[NWV], s_o[NWV][HD];
  const CachedPlace w(a, c, plan);
  const int GQ = a.n_heads / c.heads, i = w.blk / GQ, h = w.kvh * GQ + w.blk % GQ;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int grp = lane / G, gl = lane % G;
  const int qpos = w.len - a.Sq + i;
  const int k1 = w.k1 < qpos + 1 ? w.k1 : qpos + 1;
  const float slope = a.scores.slopes ? a.scores.slopes[h] : 0.f;
  float q[8], scale = a.scores.scale;
  {
    Row8<T> r;
    r.load(static_cast<const T*>(a.q.p) + w.b * a.q.batch + i * a.q.token + h * a.q.head + 8 * gl);
    float big = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      q[j] = r.get(j);
      big = fmaxf(big, fabsf(q[j]));
    }
    // a row whose sums of products with codes might pass fp32: 2^-32 of it, the same for
    // all of its lanes
    if (__builtin_expect(__ballot(big > 0x1p100f) != 0, 0)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] *= 0x1p-32f;
      scale *= 0x1p32f;
    }
  }
  const long long head = static_cast<long long>(w.b) * c.heads + w.kvh;
  const char* kc = static_cast<const char*>(c.k) + head * c.max_seq * (HD * BITS / 8) + gl * BITS;
  const char* vc = static_cast<const char*>(c.v) + head * c.max_seq * (HD * BITS / 8) + gl * BITS;
  const long long sbase = (head * (HD / kKvGroup) + gl / 4) * c.max_seq;
  const uint16_t* ks = static_cast<const uint16_t*>(c.k_scale) + sbase;
  const uint16_t* vs = static_cast<const uint16_t*>(c.v_scale) + sbase;
  const uint8_t* valid = c.valid ? c.valid + static_cast<long long>(w.b) * c.max_seq : nullptr;
  constexpr int W = BITS / 4;                  // words of 8 codes
  auto codes = [&](const uint32_t (&v)[W], float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t code = BITS == 8 ? (v[j / 4 % W] >> (8 * (j % 4))) & 255u : (v[0] >> (4 * j)) & 15u;
      x[j] = static_cast<float>(static_cast<int>(code) - OFF);
    }
  };
  // o is in units of 1 / fit: 1, or 2^32 once the group has met a scale above 2^90, whose
  // sums might pass fp32
  float m = -INFINITY, l = 0.f, o[8], fit = 1.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = 0.f;
  // U keys a lane group, their rows loaded together (keys past the end read the
  // chunk's first)
  constexpr int U = 4;
  for (int key0 = w.k0 + wave * KPW + grp; key0 < k1; key0 += U * NG) {
    uint32_t kr[U][W], vr[U][W];
    uint16_t kscale[U], vscale[U];
    uint8_t on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key = key0 + u * NG < k1 ? key0 + u * NG : w.k0;
      const long long row = static_cast<long long>(key) * (HD * BITS / 8);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        kr[u][j] = reinterpret_cast<const uint32_t*>(kc + row)[j];
        vr[u][j] = reinterpret_cast<const uint32_t*>(vc + row)[j];
      }
      kscale[u] = ks[key];
      vscale[u] = vs[key];
      on[u] = valid ? valid[key] : 1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int key = key0 + u * NG;
      float kx[8], vx[8], s = 0.f;
      codes(kr[u], kx);
      codes(vr[u], vx);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(q[j], kx[j], s);
      s *= bf16_value(kscale[u]);
#pragma unroll
      for (int off = G / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
      if (key >= k1 || !on[u]) continue;       // the same for the whole lane group
      s = modify_score(s * scale, a.scores.softcap, slope, static_cast<float>(qpos - key));
      const float mn = fmaxf(m, s);
      float sv = bf16_value(vscale[u]) * fit;
      if (__builtin_expect(sv > 0x1p90f && fit == 1.f, 0)) {
        fit = 0x1p-32f;
        sv *= fit;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] *= fit;
      }
      const float corr = m == mn ? 1.f : expf(m - mn), p = s == -INFINITY ? 0.f : expf(s - mn);
      l = l * corr + p;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = o[j] * corr + p * sv * vx[j];
      m = mn;
    }
  }
  // the lane groups' outputs, divided by their sums before they are joined
  const float own = over_sum(l) * (fit == 1.f ? 1.f : 0x1p32f);
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] *= own;
#pragma unroll
  for (int off = G; off < 64; off <<= 1) {
    const float mo = __shfl_xor(m, off, 64), lo = __shfl_xor(l, off, 64);
    const float mm = fmaxf(m, mo);
    const float w0 = l * (m == -INFINITY ? 0.f : expf(m - mm));
    const float w1 = lo * (mo == -INFINITY ? 0.f : expf(mo - mm));
    l = w0 + w1;
    m = mm;
    const float inv = over_sum(l);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = o[j] * (w0 * inv) + __shfl_xor(o[j], off, 64) * (w1 * inv);
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
  for (int x = 0; x < NWV; ++x) M = fmaxf(M, s_m[x]);
  float f[NWV];
  for (int x = 0; x < NWV; ++x) {
    f[x] = s_l[x] * (s_m[x] == -INFINITY ? 0.f : expf(s_m[x] - M));
    L += f[x];
  }
  const float inv = over_sum(L);
  for (int x = 0; x < NWV; ++x) O += s_o[x][ch] * (f[x] * inv);
  if (plan.nsplit == 1) {
    cached_out<T>(a, c, w.b, w.kvh, w.blk)[ch] = from_f32<T>(O);
    return;
  }
  float* part = cached_part<HD>(a, c, plan, w.b, w.kvh, w.blk, w.split);
  part[2 + ch] = O;
  if (ch == 0) {
    part[0] = M * kLog2e;
    part[1] = L;
  }
}

// ------------------------------------------------------------ 16-bit: MFMA
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Sum over the NG lanes n that share a row (they hold its groups), in each of them.
template <int NG>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (NG >= 2)
    v += dpp_or_zero<0xB1, 0xf>(v);   // lanes 1 0 3 2
  if constexpr (NG == 4)
    v += dpp_or_zero<0x4E, 0xf>(v);   // lanes 2 3 0 1
  return v;
}

// BYTES bytes as 32-bit words (a lone byte or half word zero-extended).
template <int BYTES>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (BYTES == 1) w[0] = *reinterpret_cast<const uint8_t*>(p);
  else if constexpr (BYTES == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
  else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
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

// Workgroup = one row block of a key head and one chunk of the keys, its 4 or 8 wavefronts
// taking tiles of 32 keys in turn; no LDS and no barrier before the end.  Codes become
// fp16 operands of v_mfma_f32_16x16x32 by bit operations alone: code bits in the low
// bits of an fp16 are the subnormal code * 2^-24 (in bits 4-7: 16 code * 2^-24), which
// the instruction multiplies exactly.  Columns n of a product are (query row n / NG,
// channel group n % NG), NG = HD / 32:
//  S[key][n]: A = K codes, a lane (key row m, lane / 16 = g) holding HD / 4 consecutive
//    channels, which lie in one group; B = the query, zero outside the column's group;
//    the codes' offset 2^(BITS - 1) is taken off the sums' start.  So a lane has the sums
//    of its group for 8 keys, multiplies by the group's K scales and adds the NG lanes of
//    its row.  Rows 4 g + r of product u are keys 8 g + 4 u + r.
//  O[ch][n] += V codes * w, the codes' offset taken off them first (a packed fp16
//    addition, exact; taken off the sums it would leave errors of an offset times w).
//    w = exp2(score - m) * V scale of the column's group, rounded to fp16 after division
//    by a power of two above the largest weight at the last look and at least an eighth
//    of any since, and times 2^8 (at most 2^11, and 2^15 where the power would pass 2^126, so
//    that what falls below fp16's smallest normal is 2^-21 of the largest weight or less; in units of the largest scale a value
//    of no weight would take the bits of all others).  The 8 keys whose scores a lane
//    holds are the 8 k slots of its B operand: w needs no exchange.  A row m of product i
//    is channel (HD / 16) m + i, a lane reading HD / 16 channels of 8 keys.  A lane's own
//    column counts where the channel's group is the column's.
// The query is divided by a power of two as well (largest element to 2^14), so that of
// bf16 and fp16 rows only elements below 2^-24 of the largest lose bits in fp16.  The
// maximum m moves lazily (by more than 2^8).
// The tile being worked on and its successor, which arrives meanwhile, are both in
// registers.
// Heads with more rows than a set of columns holds (4 of 128 channels) take more
// workgroups, which read the same codes again, mostly from cache; two sets in one
// workgroup need 256 registers and gain nothing (16 sequences of 4000 keys, 32/4 heads,
// 4 bits: 21.8 us a set each, 23.6 two; 8 bits 29.1 and 43.0).
// Measured, launches one after the other: 32 sequences of 8190 keys, 32/8 heads of 128, 4
// bits, 62 us (4.9 TB/s; a large copy reaches 4.8; 270 vector instructions per tile),
// capped 73 (300); 4 of 8000 keys, 32 heads, 8 bits, 58 us (4.8 TB/s).  Ragged, capped, the
// vector units work 73% of the time that CUs hold work, the matrix cores 12%.

// Wavefronts per SIMD that the registers of a tile, its successor and O leave room for.
constexpr int cached_waves(int hd, int bits) { return hd == 128 ? (bits == 4 ? 3 : 2) : hd == 64 ? 3 : 4; }

template <typename T, int HD, int BITS, bool CAP, int NWV>
__global__ __launch_bounds__(64 * NWV) __attribute__((amdgpu_waves_per_eu(cached_waves(HD, BITS), cached_waves(HD, BITS))))
void k_cached_mfma(gm_cached_attention a, gm_kv_cache c, CachedPlan plan) {
  constexpr int OFF = 1 << (BITS - 1), KB = 32;
  constexpr int NG = HD / kKvGroup, RB = 16 / NG;   // groups, rows per block
  constexpr int KD = HD * BITS / 128;               // words of a lane's K chunk
  constexpr int VB = HD * BITS / 128, VD = VB < 4 ? 1 : VB / 4;   // bytes, words of its V chunk
  constexpr int NI = HD / 16;                       // products of O
  constexpr float kTau = 8.f, kTiny = 1.f / 16777216.f;           // 2^-24
  __shared__ float s_m[NWV][RB], s_l[NWV][RB], s_o[NWV][RB][HD + 1];
  const CachedPlace w(a, c, plan);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4, t = n % NG;
  const int r = w.blk * RB + n / NG;                // this column's query row
  const bool row_ok = r < plan.rows;
  const int GQ = a.n_heads / c.heads, rr = row_ok ? r : 0, i = rr / GQ, h = w.kvh * GQ + rr % GQ;
  // (columns past the last row repeat row 0 and are not used)
  const int qpos = w.len - a.Sq + i, open = w.len - a.Sq;   // every row sees keys up to `open`
  const float slope2 = a.scores.slopes ? a.scores.slopes[h] * kLog2e : 0.f;

  // ---- the query as B operands: k step st, slots 2 d and 2 d + 1 hold the channels whose
  // codes the unpacking below puts there
  f16x8 qf[NG];
  float c0, up;                                     // start of the sums of S; part of their unit
  float c2 = CAP ? a.scores.scale * (2.f * kLog2e) / a.scores.softcap : a.scores.scale * kLog2e;
  {
    constexpr int NC = HD / 4;
    float x[NC], big = 0.f, sum = 0.f;
    const T* q = static_cast<const T*>(a.q.p) + w.b * a.q.batch + i * a.q.token + h * a.q.head + NC * g;
#pragma unroll
    for (int j = 0; j < NC / 8; ++j) {
      Row8<T> v;
      v.load(q + 8 * j);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * j + e] = v.get(e);
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) big = fmaxf(big, fabsf(x[j]));
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    const int ex = big > 0.f && big < INFINITY ? static_cast<int>(__float_as_uint(big) >> 23) - 127 : 0;
    const bool mine = t == g * NG / 4;
#pragma unroll
    for (int st = 0; st < NG; ++st)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // slot j of word j / 2: nibbles j / 2 and j / 2 + 4, or bytes j
        const int ch = BITS == 4 ? j / 2 + 4 * (j % 2) : j;
        const float v = mine ? ldexpf(x[8 * st + ch], 14 - ex) : 0.f;
        const float sixteen = BITS == 4 && (j / 2) % 2 ? 0.0625f : 1.f;
        const _Float16 f = static_cast<_Float16>(v * sixteen);
        qf[st][j] = f;
        sum += static_cast<float>(f) * (1.f / sixteen);
      }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    c0 = -static_cast<float>(OFF) * kTiny * sum;
    // the sums' unit 2^24 / 2^(14 - ex); of rows near the ends of fp32 a part goes
    // to the K scales
    const int part = 10 + ex > 90 ? 10 + ex - 90 : 10 + ex < -90 ? 100 + ex : 0;
    up = ldexpf(1.f, part);
    c2 = ldexpf(c2, 10 + ex - part);
  }
  const float capc = a.scores.softcap * kLog2e;

  const long long head = static_cast<long long>(w.b) * c.heads + w.kvh;
  const char* kc = static_cast<const char*>(c.k) + head * c.max_seq * (HD * BITS / 8) +
                   (8 * (n >> 2) + (n & 3)) * (HD * BITS / 8) + 4 * KD * g;
  const char* vc = static_cast<const char*>(c.v) + head * c.max_seq * (HD * BITS / 8) +
                   8 * g * (HD * BITS / 8) + VB * n;
  const uint16_t* ks = static_cast<const uint16_t*>(c.k_scale) + (head * NG + t) * c.max_seq + 8 * g;
  const uint16_t* vs = static_cast<const uint16_t*>(c.v_scale) + (head * NG + t) * c.max_seq + 8 * g;
  const uint8_t* valid = c.valid ? c.valid + static_cast<long long>(w.b) * c.max_seq + 8 * g : nullptr;

  struct Tile {
    uint32_t k[2][KD], v[8][VD];
    u32x4 ks, vs;
    u32x2 valid;
  };
  auto fetch = [&](int kb, Tile& x) {
    const long long row = static_cast<long long>(kb) * (HD * BITS / 8);
#pragma unroll
    for (int u = 0; u < 2; ++u) load_words<4 * KD>(kc + row + 4 * u * (HD * BITS / 8), x.k[u]);
    x.ks = *reinterpret_cast<const u32x4*>(ks + kb);
#pragma unroll
    for (int j = 0; j < 8; ++j) load_words<VB>(vc + row + j * (HD * BITS / 8), x.v[j]);
    x.vs = *reinterpret_cast<const u32x4*>(vs + kb);
    if (valid) x.valid = *reinterpret_cast<const u32x2*>(valid + kb);
  };

  float m = -INFINITY, l = 0.f;
  // the largest weight p * V scale at the last look; one over the power of two above it
  // (2^-119 to 2^126, so that 2^8 times this is finite)
  float peak = 0.f, inv_unit = __uint_as_float((127u + 119) << 23);
  auto unit_of = [](float inv) { return __uint_as_float((254u << 23) - __float_as_uint(inv)); };
  f32x4 o[NI];
#pragma unroll
  for (int e = 0; e < NI; ++e) o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  f16x8 off[2];                                     // the codes' offset, in units of 2^-24 and 2^-20
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    off[0][j] = static_cast<_Float16>(OFF * kTiny);
    off[1][j] = static_cast<_Float16>(OFF * kTiny * (BITS == 4 ? 16.f : 1.f));
  }

  const bool wide = __ballot(up != 1.f) != 0;
  auto step = [&](int kb, const Tile& x) {
    // ---- scores of 8 keys
    float s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 acc = {c0, c0, c0, c0};
#pragma unroll
      for (int st = 0; st < NG; ++st) {
        u32x4 f;
        if constexpr (BITS == 4) {
          const uint32_t lo = x.k[u][st], hi = lo >> 8;
          f[0] = lo & 0x000f000fu;
          f[1] = lo & 0x00f000f0u;
          f[2] = hi & 0x000f000fu;
          f[3] = hi & 0x00f000f0u;
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d)
            f[d] = __builtin_amdgcn_perm(0u, x.k[u][2 * st + d / 2], d % 2 ? 0x0c030c02u : 0x0c010c00u);
        }
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, f), qf[st], acc, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[4 * u + e] = acc[e];
    }
    float sk[8], sv[8], most = 0.f, top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sk[j] = __uint_as_float(j % 2 ? x.ks[j / 2] & 0xffff0000u : x.ks[j / 2] << 16);
      sv[j] = __uint_as_float(j % 2 ? x.vs[j / 2] & 0xffff0000u : x.vs[j / 2] << 16);
    }
    if (wide) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sk[j] *= up;
    }
    const float dist = static_cast<float>(qpos - kb - 8 * g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float y = group_sum<NG>(s[j] * sk[j]) * c2;
      if constexpr (CAP) y = fmaf(-2.f * capc, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y) + 1.f), capc);
      s[j] = fmaf(-slope2, dist - static_cast<float>(j), y);
    }
    if (valid || kb + KB - 1 > open || kb + KB > w.k1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        bool ok = kb + 8 * g + j <= qpos && kb + 8 * g + j < w.k1;
        if (valid) ok = ok && ((x.valid[j / 4] >> (8 * (j % 4))) & 255u) != 0;
        s[j] = ok ? s[j] : -INFINITY;
        sv[j] = ok ? sv[j] : 0.f;                   // (it may be NaN)
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, s[j]);
    float f = 1.f;
    const bool moved = __ballot(top > m + kTau) != 0;
    if (moved) {
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float mn = fmaxf(m, top);
      f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= f;
      m = mn;
    }
    // ---- weights
    const float msub = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[j] = __builtin_amdgcn_exp2f(s[j] - msub);
      l += s[j];
      most = fmaxf(most, s[j] * sv[j]);
    }
    // a weight past 8 times that, or a new maximum, under which the old ones count for less
    if (moved || __ballot(most > 8.f * peak)) {
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      peak = fminf(fmaxf(peak * f, most), 3.4028234e38f);   // (a product past fp32: its largest)
      const uint32_t e = __float_as_uint(peak) >> 23;
      f *= unit_of(inv_unit);                       // (old / new unit alone may pass fp32)
      inv_unit = __uint_as_float((e < 7 ? 246 : e > 252 ? 1 : 253 - e) << 23);
      f *= inv_unit;
#pragma unroll
      for (int e2 = 0; e2 < NI; ++e2) o[e2] *= f;
    }
    f16x8 wf;
#pragma unroll
    for (int j = 0; j < 8; ++j) wf[j] = static_cast<_Float16>(s[j] * (sv[j] * (256.f * inv_unit)));
    // ---- O += V w: word j of product e holds keys 2 j (low half) and 2 j + 1
    if constexpr (BITS == 4) {
#pragma unroll
      for (int half = 0; half < (NI + 3) / 4; ++half) {
        u32x4 lo, hi;                               // 4 channels of 8 keys, and shifted down by two
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lo[j] = __builtin_amdgcn_perm(x.v[2 * j + 1][0], x.v[2 * j][0], half ? 0x07060302u : 0x05040100u);
          hi[j] = lo[j] >> 8;
        }
#pragma unroll
        for (int e = 0; e < (NI < 4 ? NI : 4); ++e) {
          u32x4 f;
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = (e < 2 ? lo[j] : hi[j]) & (e % 2 ? 0x00f000f0u : 0x000f000fu);
          o[4 * half + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              __builtin_bit_cast(f16x8, f) - off[e % 2], wf, o[4 * half + e], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < NI; ++e) {
        u32x4 f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          f[j] = __builtin_amdgcn_perm(x.v[2 * j + 1][e / 4], x.v[2 * j][e / 4],
                                       0x0c040c00u + 0x00010001u * (e % 4));
        o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, f) - off[0], wf, o[e], 0, 0, 0);
      }
    }
  };
  // ---- two tiles in turn, one being worked on while the other arrives
  Tile x0, x1;
  int kb = w.k0 + KB * wave;
  if (kb < w.k1) fetch(kb, x0);
  while (kb < w.k1) {
    if (kb + NWV * KB < w.k1) fetch(kb + NWV * KB, x1);
    step(kb, x0);
    kb += NWV * KB;
    if (kb >= w.k1) break;
    if (kb + NWV * KB < w.k1) fetch(kb + NWV * KB, x0);
    step(kb, x1);
    kb += NWV * KB;
  }
  // ---- the wavefront's normalised output: rows 4 g + e of product x are channels
  // NI (4 g + e) + x, of group g NG / 4
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (t == g * NG / 4) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int x = 0; x < NI; ++x) {
        const float unit = BITS == 4 && x % 2 ? 4096.f : 65536.f;   // 2^20 or 2^24, over 2^8
        s_o[wave][n / NG][NI * (4 * g + e) + x] =
            l == 0.f ? 0.f : (o[x][e] * unit * inv) * unit_of(inv_unit);
      }
  }
  if (t == 0 && g == 0) {
    s_m[wave][n / NG] = m;
    s_l[wave][n / NG] = l;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < RB * HD; e += 64 * NWV) {
    const int ch = e % HD, row = e / HD, gr = w.blk * RB + row;
    if (gr >= plan.rows) break;
    float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
    for (int x = 0; x < NWV; ++x) M = fmaxf(M, s_m[x][row]);
    float f[NWV];
#pragma unroll
    for (int x = 0; x < NWV; ++x) {
      f[x] = s_m[x][row] == -INFINITY && s_l[x][row] == 0.f
                 ? 0.f : s_l[x][row] * __builtin_amdgcn_exp2f(s_m[x][row] - M);
      L += f[x];
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;   // (before the products, which might pass fp32)
#pragma unroll
    for (int x = 0; x < NWV; ++x) O += f[x] == 0.f ? 0.f : f[x] * inv * s_o[x][row][ch];
    if (plan.nsplit == 1) {
      cached_out<T>(a, c, w.b, w.kvh, gr)[ch] = from_f32<T>(O);
    } else {
      float* part = cached_part<HD>(a, c, plan, w.b, w.kvh, gr, w.split);
      part[2 + ch] = O;
      if (ch == 0) {
        part[0] = M;
        part[1] = L;
      }
    }
  }
}

// The chunks of a row merged, a workgroup per row: the weights by the first wavefront,
// a lane per chunk (at most 64), then the chunks in 256 / HD parts, each in order, and
// the parts in theirs.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_cached_merge(gm_cached_attention a, gm_kv_cache c,
                                                      CachedPlan plan) {
  constexpr int PARTS = 256 / HD;
  __shared__ float s_w[64], s_o[PARTS][HD];
  const int tid = threadIdx.x, ch = tid % HD, of = tid / HD;
  int x = blockIdx.x;
  const int r = x % plan.rows;
  x /= plan.rows;
  const int kvh = x % c.heads, b = x / c.heads;
  const float* part = cached_part<HD>(a, c, plan, b, kvh, r, 0);
  constexpr int U = 8;
  float o[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int s = of + u * PARTS;
    o[u] = s < plan.nsplit ? part[s * (HD + 2) + 2 + ch] : 0.f;
  }
  if (tid < 64) {
    const bool on = tid < plan.nsplit;
    const float m = on ? part[tid * (HD + 2)] : -INFINITY, l = on ? part[tid * (HD + 2) + 1] : 0.f;
    const float M = wave_max(m);
    const float w = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f(m - M);
    const float W = wave_sum(w);
    s_w[tid] = w == 0.f ? 0.f : w / W;
  }
  __syncthreads();
  float sum = 0.f;
  for (int s0 = 0; s0 < plan.nsplit; s0 += U * PARTS) {
    if (s0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + of + u * PARTS;
        o[u] = s < plan.nsplit ? part[s * (HD + 2) + 2 + ch] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + of + u * PARTS;
      const float w = s < plan.nsplit ? s_w[s] : 0.f;
      sum += w == 0.f ? 0.f : w * o[u];
    }
  }
  s_o[of][ch] = sum;
  __syncthreads();
  if (of) return;
#pragma unroll
  for (int p = 1; p < PARTS; ++p) sum += s_o[p][ch];
  cached_out<T>(a, c, b, kvh, r)[ch] = from_f32<T>(sum);
}

}  // namespace

uint64_t attention_cached_workspace(const gm_kv_cache& c, int dtype, int B, int Sq, int n_heads) {
  const CachedPlan p = cached_plan(c, dtype, B, Sq, n_heads);
  if (p.nsplit == 1) return 0;
  return static_cast<uint64_t>(B) * c.heads * p.rows * p.nsplit * (c.head_dim + 2) * sizeof(float);
}

void launch_attention_cached(const gm_cached_attention& a, hipStream_t s) {
  const gm_kv_cache& c = *a.cache;
  const CachedPlan p = cached_plan(c, a.dtype, a.B, a.Sq, a.n_heads);
  const unsigned heads = static_cast<unsigned>(a.B) * c.heads;
  const dim3 grid(heads * p.blocks, p.nsplit), block(256);
  by_cache(a.dtype, c, [&](auto t, auto hd, auto bits) {
    typedef decltype(t) T;
    constexpr int HD = decltype(hd)::value, BITS = decltype(bits)::value;
    if constexpr (std::is_same<T, float>::value)
      hipLaunchKernelGGL((k_cached_rows<T, HD, BITS>), grid, block, 0, s, a, c, p);
    else {
      auto go = [&](auto cap, auto waves) {
        constexpr int NWV = decltype(waves)::value;
        hipLaunchKernelGGL((k_cached_mfma<T, HD, BITS, decltype(cap)::value, NWV>), grid, dim3(64 * NWV), 0, s,
                           a, c, p);
      };
      auto width = [&](auto cap) {
        if (p.waves == 8) go(cap, std::integral_constant<int, 8>());
        else go(cap, std::integral_constant<int, 4>());
      };
      if (a.scores.softcap > 0.f) width(std::true_type());
      else width(std::false_type());
    }
    if (p.nsplit > 1)
      hipLaunchKernelGGL((k_cached_merge<T, HD>), dim3(heads * p.rows), block, 0, s, a, c, p);
  });
}

}  // namespace gm
