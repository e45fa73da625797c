// AdamW over a list of tensors, optimizer states in 32 or in 8 bits.
//
// A wave takes a run of one tensor's 256-element blocks, four consecutive
// elements a lane; the list travels in the kernel's arguments, as many tensors
// a launch as those hold.  An element's arithmetic is rounded after every
// operation (no fused multiply-add), so that the states, and with 8 bits the
// codes that their rounding picks, do not depend on how a compiler contracts
// it.
//
// Bound by HBM: 32-bit states with fp32 gradients and a bf16 copy move 30 bytes
// a weight (the ResNet18's 62 tensors, 11.2 M weights: 67 us, 5.0 TB/s), 8-bit
// states with bf16 gradients and the copy 16 (134 M weights: 396 us, 5.4 TB/s); a
// large copy reaches 5.1 TB/s.  Two small tensors take 4 us.  Blocks of 256 share
// a scale so that a wave finds their largest value without LDS, and four
// elements a lane make one 16-byte access of the fp32 arrays.
#include <algorithm>
#include <cmath>

#include "kernels.hpp"

namespace ekya {
namespace {

constexpr int AD_NT = 256, AD_WAVES = AD_NT / 64;
constexpr int AD_BLOCK = 256;              // elements that share a scale
constexpr int AD_RUN = 2;                  // blocks of a wave
constexpr int AD_ITEM = AD_BLOCK * AD_RUN; // elements of a wave
constexpr long long AD_MOST = 1 << 24;     // waves of a launch
constexpr uint64_t AD_GOLDEN = 0x9E3779B97F4A7C15ull, AD_TAG = 0xD1B54A32D192ED03ull;

template <int BITS> struct AdEntry;
template <> struct AdEntry<32> {
  float* w;
  const void* g;
  float *m, *v;
  bf16* low;
  long long n;
  float keep;      // 1 - lr * weight_decay
  uint32_t item0;  // the entry's first wave
};
template <> struct AdEntry<8> {
  float* w;
  const void* g;
  uint8_t *m, *v;
  bf16* low;
  float* scale;
  long long n;
  float keep;
  uint32_t item0;
  uint32_t block0;  // the entry's first 256-element block, from the launch's
};

struct AdOpts {
  float b1, c1, b2, c2, eps;  // c = 1 - b
  float rate, root;           // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float lr;
  double log1, log2;          // natural logarithms of the betas
  const int64_t* step;        // or null: rate and root as given
  uint64_t seed;              // with the step's part in it where step is null
};

// Kernel arguments stay below 4 KB with the runtime's own.
template <int BITS> struct AdArgs {
  static constexpr int MOST = (3840 - (int)sizeof(AdOpts) - 16) / (int)sizeof(AdEntry<BITS>);
  AdEntry<BITS> t[MOST];
  AdOpts o;
  uint64_t base;  // 256-element blocks before the launch's first
  int count;
  uint32_t items;
};

// Four elements from p, `cnt` of them there (the others: 0).
template <bool FULL> __device__ __forceinline__ void ad_load(const float* p, int cnt, float (&v)[4]) {
  if constexpr (FULL) return load4(p, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < cnt ? p[i] : 0.f;
}
template <bool FULL> __device__ __forceinline__ void ad_load(const bf16* p, int cnt, float (&v)[4]) {
  if constexpr (FULL) return load4(p, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < cnt ? (float)p[i] : 0.f;
}
template <bool FULL> __device__ __forceinline__ uint32_t ad_load(const uint8_t* p, int cnt) {
  if constexpr (FULL) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) v |= i < cnt ? (uint32_t)p[i] << (8 * i) : 0u;
  return v;
}
template <bool FULL, typename T>
__device__ __forceinline__ void ad_store(T* p, int cnt, const float (&v)[4]) {
  if constexpr (FULL) return store4(p, v);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < cnt) p[i] = from_f<T>(v[i]);
}
template <bool FULL> __device__ __forceinline__ void ad_store(uint8_t* p, int cnt, uint32_t v) {
  if constexpr (FULL) {
    *reinterpret_cast<uint32_t*>(p) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < cnt) p[i] = (uint8_t)(v >> (8 * i));
}

__device__ __forceinline__ void ad_decode(uint32_t code, float scale, float (&v)[4], bool e5m2) {
  if (e5m2) {  // the upper byte of an fp16
    v[0] = __builtin_amdgcn_cvt_f32_bf8(code, 0);
    v[1] = __builtin_amdgcn_cvt_f32_bf8(code, 1);
    v[2] = __builtin_amdgcn_cvt_f32_bf8(code, 2);
    v[3] = __builtin_amdgcn_cvt_f32_bf8(code, 3);
  } else {
    v[0] = __builtin_amdgcn_cvt_f32_fp8(code, 0);
    v[1] = __builtin_amdgcn_cvt_f32_fp8(code, 1);
    v[2] = __builtin_amdgcn_cvt_f32_fp8(code, 2);
    v[3] = __builtin_amdgcn_cvt_f32_fp8(code, 3);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] *= scale;
}

// Output `i` (from 0) of the SplitMix64 stream that starts at `start`.
__device__ __forceinline__ uint64_t splitmix(uint64_t start, uint64_t i) {
  uint64_t z = start + (i + 1) * AD_GOLDEN;
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

// Codes of four magnitudes, MANT mantissa bits and exponents biased by BIAS,
// each rounded up with the probability of its remainder; rnd: 16 random bits
// each.  The scale is the power of two that puts the block's largest finite
// magnitude, whose bits are `most`, into [2^TOP, 2^(TOP + 1)).
template <int MANT, int BIAS, int TOP, uint32_t HIGHEST>
__device__ __forceinline__ void ad_encode(const float (&x)[4], const uint32_t (&rnd)[4], uint32_t most,
                                          uint32_t (&code)[4], float& scale) {
  constexpr int DROP = 23 - MANT;
  const int k = max((int)(most >> 23) - 127 - TOP, -126);
  scale = __uint_as_float((uint32_t)(k + 127) << 23);
  const float inv = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = fabsf(x[i]) * inv;
    const uint32_t bits = __float_as_uint(a), r = (rnd[i] << (DROP - 16)) + (1u << (DROP - 17));
    const uint32_t normal = ((bits + r) >> DROP) - ((127u - BIAS) << MANT);
    const uint32_t small = ((uint32_t)(a * (float)(1ull << (DROP + BIAS - 1 + MANT))) + r) >> DROP;
    const uint32_t c = bits >= (128u - BIAS) << 23 ? normal : small;
    code[i] = (__float_as_uint(x[i]) & 0x7F800000u) == 0x7F800000u ? 0x7Fu : min(c, HIGHEST);
  }
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

struct AdRates {
  float rate, root;
  uint64_t start;  // of the random stream
};

__device__ __forceinline__ void ad_element(const AdOpts& o, const AdRates& r, float keep, float g,
                                           float& w, float& m, float& v) {
#pragma clang fp contract(off)
  m = o.b1 * m + o.c1 * g;
  v = o.b2 * v + o.c2 * (g * g);
  const float denom = sqrtf(v) * r.root + o.eps;
  w = w * keep - r.rate * (m / denom);
}

template <bool FULL, typename G>
__device__ __forceinline__ void ad_item(const AdEntry<32>& t, const AdOpts& o, const AdRates& r,
                                        uint64_t, long long first, int lane) {
  float w[AD_RUN][4], g[AD_RUN][4], m[AD_RUN][4], v[AD_RUN][4];
  long long at[AD_RUN];
  int cnt[AD_RUN];
#pragma unroll
  for (int u = 0; u < AD_RUN; ++u) {
    at[u] = first + u * AD_BLOCK + lane * 4;
    cnt[u] = FULL ? 4 : (int)max(0LL, min(4LL, t.n - at[u]));
    ad_load<FULL>(t.w + at[u], cnt[u], w[u]);
    ad_load<FULL>((const G*)t.g + at[u], cnt[u], g[u]);
    ad_load<FULL>(t.m + at[u], cnt[u], m[u]);
    ad_load<FULL>(t.v + at[u], cnt[u], v[u]);
  }
#pragma unroll
  for (int u = 0; u < AD_RUN; ++u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) ad_element(o, r, t.keep, g[u][i], w[u][i], m[u][i], v[u][i]);
    ad_store<FULL>(t.w + at[u], cnt[u], w[u]);
    ad_store<FULL>(t.m + at[u], cnt[u], m[u]);
    ad_store<FULL>(t.v + at[u], cnt[u], v[u]);
    if (t.low) ad_store<FULL>(t.low + at[u], cnt[u], w[u]);
  }
}

template <bool FULL, typename G>
__device__ __forceinline__ void ad_item(const AdEntry<8>& t, const AdOpts& o, const AdRates& r,
                                        uint64_t block, long long first, int lane) {
  float w[AD_RUN][4], g[AD_RUN][4], sm[AD_RUN], sv[AD_RUN];
  uint32_t mc[AD_RUN], vc[AD_RUN];
  long long at[AD_RUN];
  int cnt[AD_RUN];
#pragma unroll
  for (int u = 0; u < AD_RUN; ++u) {
    const long long from = first + u * AD_BLOCK;
    at[u] = from + lane * 4;
    cnt[u] = FULL ? 4 : (int)max(0LL, min(4LL, t.n - at[u]));
    ad_load<FULL>(t.w + at[u], cnt[u], w[u]);
    ad_load<FULL>((const G*)t.g + at[u], cnt[u], g[u]);
    mc[u] = ad_load<FULL>(t.m + at[u], cnt[u]);
    vc[u] = ad_load<FULL>(t.v + at[u], cnt[u]);
    const bool there = FULL || from < t.n;
    sm[u] = there ? t.scale[from / AD_BLOCK * 2] : 0.f;
    sv[u] = there ? t.scale[from / AD_BLOCK * 2 + 1] : 0.f;
  }
#pragma unroll
  for (int u = 0; u < AD_RUN; ++u) {
    float m[4], v[4];
    ad_decode(mc[u], sm[u], m, false);
    ad_decode(vc[u], sv[u], v, true);
    uint32_t mm = 0, mv = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (FULL || i < cnt[u]) {
        ad_element(o, r, t.keep, g[u][i], w[u][i], m[i], v[i]);
        mm = max(mm, finite_bits(m[i]));
        mv = max(mv, finite_bits(v[i]));
      }
    }
    mm = wave_max(mm);
    mv = wave_max(mv);
    const uint64_t z = splitmix(r.start, (block + u) * (AD_BLOCK / 4) + lane);
    uint32_t up[4], down[4], cm[4], cv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      up[i] = (uint32_t)(z >> (16 * i)) & 0xFFFFu;
      down[i] = 0xFFFFu - up[i];
    }
    ad_encode<3, 7, 7, 0x7Eu>(m, up, mm, cm, sm[u]);
    ad_encode<2, 15, 14, 0x7Bu>(v, down, mv, cv, sv[u]);
    uint32_t pm = 0, pv = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pm |= (cm[i] | (m[i] < 0.f ? 0x80u : 0u)) << (8 * i);
      pv |= max(cv[i], v[i] > 0.f ? 1u : 0u) << (8 * i);
    }
    ad_store<FULL>(t.w + at[u], cnt[u], w[u]);
    ad_store<FULL>(t.m + at[u], cnt[u], pm);
    ad_store<FULL>(t.v + at[u], cnt[u], pv);
    if (t.low) ad_store<FULL>(t.low + at[u], cnt[u], w[u]);
    if (lane == 0 && (FULL || first + u * AD_BLOCK < t.n)) {
      float* s = t.scale + (first / AD_BLOCK + u) * 2;
      s[0] = sm[u];
      s[1] = sv[u];
    }
  }
}

__device__ __forceinline__ bool on(const void* p, int n) {
  return reinterpret_cast<uintptr_t>(p) % n == 0;
}

template <int BITS, typename G>
__global__ __launch_bounds__(AD_NT) void adamw_kernel(AdArgs<BITS> a) {
  const int lane = threadIdx.x & 63;
  const uint32_t item = blockIdx.x * AD_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= a.items) return;
  int lo = 0, hi = a.count - 1;  // the last entry that starts at or before the item
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.t[mid].item0 <= item) lo = mid; else hi = mid - 1;
  }
  const AdEntry<BITS>& t = a.t[lo];
  AdRates r{a.o.rate, a.o.root, a.o.seed};
  if (a.o.step) {
    const int64_t step = max((int64_t)1, *a.o.step);
    r.rate = a.o.lr / -expm1f((float)(a.o.log1 * (double)step));
    r.root = 1.f / sqrtf(-expm1f((float)(a.o.log2 * (double)step)));
    r.start += (uint64_t)step * AD_TAG;
  }
  const long long first = (long long)(item - t.item0) * AD_ITEM;
  uint64_t block = 0;
  constexpr int SB = BITS == 32 ? 16 : 4;  // bytes of four states
  if constexpr (BITS == 8) block = a.base + t.block0 + first / AD_BLOCK;
  const bool full = first + AD_ITEM <= t.n && on(t.w, 16) && on(t.g, 4 * sizeof(G)) &&
                    on(t.m, SB) && on(t.v, SB) && on(t.low, 8);
  if (full)
    ad_item<true, G>(t, a.o, r, block, first, lane);
  else
    ad_item<false, G>(t, a.o, r, block, first, lane);
}

template <int BITS> void ad_fill(AdEntry<BITS>& e, const AdamwTensor& t, long long from, long long n) {
  e.w = t.w + from;
  e.m = (decltype(e.m))t.m + from;
  e.v = (decltype(e.v))t.v + from;
  e.low = t.low ? (bf16*)t.low + from : nullptr;
  e.n = n;
  if constexpr (BITS == 8) e.scale = t.scale + from / AD_BLOCK * 2;
}

template <int BITS, typename G>
hipError_t ad_run(const AdamwTensor* t, int count, const AdOpts& o, double lr, hipStream_t st) {
  AdArgs<BITS> a;
  a.o = o;
  a.base = 0;
  a.count = 0;
  a.items = 0;
  uint64_t blocks = 0;  // of the list so far
  auto flush = [&]() {
    if (a.count) {
      hipLaunchKernelGGL((adamw_kernel<BITS, G>), dim3((a.items + AD_WAVES - 1) / AD_WAVES),
                         dim3(AD_NT), 0, st, a);
      EKYA_HIP(hipGetLastError());
    }
    a.base = blocks;
    a.count = 0;
    a.items = 0;
    return hipSuccess;
  };
  for (int i = 0; i < count; ++i)
    for (long long from = 0; from < t[i].n;) {
      if (a.count == a.MOST || a.items == AD_MOST) EKYA_HIP(flush());
      const long long n = std::min<long long>(t[i].n - from, (AD_MOST - a.items) * AD_ITEM);
      AdEntry<BITS>& e = a.t[a.count++];
      ad_fill(e, t[i], from, n);
      e.g = (const G*)t[i].g + from;
      e.keep = (float)(1.0 - lr * t[i].weight_decay);
      e.item0 = a.items;
      if constexpr (BITS == 8) e.block0 = (uint32_t)(blocks - a.base);
      a.items += (uint32_t)cdivl(n, AD_ITEM);
      blocks += cdivl(n, AD_BLOCK);
      from += n;
    }
  return flush();
}

}  // namespace

hipError_t adamw_step(const AdamwTensor* t, int count, int grad_dt, int bits, double lr,
                      double beta1, double beta2, double eps, long long step,
                      const int64_t* step_device, uint64_t seed, hipStream_t st) {
  AdOpts o;
  o.b1 = (float)beta1;
  o.c1 = (float)(1 - beta1);
  o.b2 = (float)beta2;
  o.c2 = (float)(1 - beta2);
  o.eps = (float)eps;
  o.lr = (float)lr;
  o.log1 = log(beta1);
  o.log2 = log(beta2);
  o.step = step_device;
  o.seed = seed;
  o.rate = o.root = 0.f;
  if (!step_device) {
    o.rate = (float)(lr / -expm1(step * o.log1));
    o.root = (float)(1 / sqrt(-expm1(step * o.log2)));
    o.seed += (uint64_t)step * AD_TAG;
  }
  if (bits == 8)
    return grad_dt == DT_F32 ? ad_run<8, float>(t, count, o, lr, st) : ad_run<8, bf16>(t, count, o, lr, st);
  return grad_dt == DT_F32 ? ad_run<32, float>(t, count, o, lr, st) : ad_run<32, bf16>(t, count, o, lr, st);
}

}  // namespace ekya
