// Group norm with an activation over channels-last activations, forward and
// backward.
//
//   xhat = (x - mean) rstd,  u = xhat gamma + beta,  y = act(u)
//   g = dy act'(u),  dbeta = sum g,  dgamma = sum g xhat,  h = g gamma,
//   dx = rstd (h - avg h - xhat avg(h xhat)), averages over the (sample, group)
//
// Bound by HBM: 2 (3) elements of traffic for each of x.  Where a block can
// hold the pixels of whole groups in registers, one launch reads x (and dy)
// once: 128 x 3136 x 64 bf16, 32 groups, forward 31 us (103 MB; a copy of as much
// takes 20), backward 56 us with the launch that adds up the parameters'
// gradients (154 MB; 30); one frame of 49 x 512 takes 6 us.  A block's loads,
// sums and stores follow one another, and all blocks run at once, so reading
// and writing hardly overlap: that is what is left.
//
// Else (long samples, groups of many channels, channel counts or addresses
// off 16 bytes) x is read twice: partial statistics, coefficients, results.  A
// block takes a range of pixels of one sample and up to 64 16-byte units of its
// channels; a thread keeps one unit's channels and walks the pixels.  Sums are
// kept per channel, whatever the group size (groups of 3 or 10 channels straddle
// the units), and folded into groups by the coefficient kernels.  Means and
// squared deviations are merged pairwise (Chan, Golub and LeVeque), so that a
// mean far from zero costs no digits.  128 x 3136 x 64 in one group: 41 us forward,
// 62 backward; 19 x 1147 x 120 fp32 in groups of 10 backward 21 us.
#include <algorithm>
#include <climits>
#include <numeric>

#include "act.hpp"
#include "kernels.hpp"

namespace ekya {
namespace {

constexpr int GN_NT = 256;  // threads of a block
constexpr int GN_R = 8;     // pixels a thread has in flight

// E consecutive elements of a channel run: a 16-byte unit, or one element
// where channels or addresses allow no units.
template <typename T, int E> struct GnUnit {
  uint4 u;
  __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[E]) const {
    Unit<T> t;
    t.u = u;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = to_f(t.e[e]);
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[E]) {
    Unit<T> t;
#pragma unroll
    for (int e = 0; e < E; ++e) t.e[e] = from_f<T>(v[e]);
    *reinterpret_cast<uint4*>(p) = t.u;
  }
};
// Between two passes over units in registers: the compiler would keep the first
// pass's unpacked values for the second, in twice the registers.
__device__ __forceinline__ void gn_renew(uint4& u) {
  asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
}
__device__ __forceinline__ void gn_renew(uint2& u) { asm volatile("" : "+v"(u.x), "+v"(u.y)); }
template <typename U> __device__ __forceinline__ void gn_renew(U&) {}

template <> struct GnUnit<bf16, 4> {  // 8 bytes
  uint2 u;
  __device__ __forceinline__ void load(const bf16* p) { u = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    v[0] = __uint_as_float(u.x << 16);
    v[1] = __uint_as_float(u.x & 0xFFFF0000u);
    v[2] = __uint_as_float(u.y << 16);
    v[3] = __uint_as_float(u.y & 0xFFFF0000u);
  }
  static __device__ __forceinline__ void store(bf16* p, const float (&v)[4]) { store4(p, v); }
};
template <typename T> struct GnUnit<T, 1> {
  T u;
  __device__ __forceinline__ void load(const T* p) { u = *p; }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f(u); }
  static __device__ __forceinline__ void store(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }
};

struct GnArgs {
  const void *x, *dy;
  void* out;
  const float *gamma, *beta;  // null: 1 and 0
  float *mean, *rstd;         // [N][G]
  float* part;                // [N][slots][C][2] (backward: [N][chunks][2][C])
  float* tot;                 // [N][2][C] (backward)
  float* coef;                // [N][G][2] (backward)
  float* slices;              // [GN_SLICES][2][C] (backward)
  float *dgamma, *dbeta;
  long long HW;
  int N, C, G, gs;       // gs: channels of a group
  int cu, cup, cchunks;  // units of a channel chunk, the next power of two, chunks
  int rows, chunks;      // pixels of a chunk, chunks of a sample
  int srows, slots;      // the same for a wave of the statistics pass
  float eps;
};

// A block's sample, pixel range and channel unit.
struct GnPlace {
  int n, chunk, c;     // c: the thread's first channel
  long long r0, r1;    // pixels
  int r, rpp;          // the thread's row within a pass, rows of a pass
  bool on;
};
template <int E> __device__ __forceinline__ GnPlace gn_place(const GnArgs& a) {
  GnPlace p;
  const int b = blockIdx.x, per = a.chunks * a.cchunks;
  p.n = b / per;
  const int rest = b - p.n * per;
  p.chunk = rest / a.cchunks;
  const int u = threadIdx.x & (a.cup - 1);
  p.r = threadIdx.x / a.cup;
  p.rpp = GN_NT / a.cup;
  p.c = ((rest - p.chunk * a.cchunks) * a.cu + u) * E;
  p.on = u < a.cu && p.c < a.C;
  p.r0 = (long long)p.chunk * a.rows;
  p.r1 = min(a.HW, p.r0 + a.rows);
  return p;
}

// Sums v over the threads of a block that share a channel unit, in a fixed
// order; threads of the first row return the totals.  red: GN_NT * E floats.
template <int E> __device__ __forceinline__ void gn_row_sum(float (&v)[E], float* red, int cup) {
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) red[threadIdx.x * E + e] = v[e];
  __syncthreads();
  for (int h = GN_NT / 2; h >= cup; h >>= 1) {
    if ((int)threadIdx.x < h)
#pragma unroll
      for (int e = 0; e < E; ++e) red[threadIdx.x * E + e] += red[(threadIdx.x + h) * E + e];
    __syncthreads();
  }
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = red[threadIdx.x * E + e];
}

// part[n][slot][c] = (mean, squared deviations) of a slot's pixels: a wave
// each, whose lanes keep a unit and walk its rows.  Lanes merge by shuffles,
// without a barrier (with sums over the block through LDS 128 x 3136 x 64 took 24
// us for this pass).
template <typename T, int E> __global__ __launch_bounds__(GN_NT) void gn_stats_kernel(GnArgs a) {
  constexpr int S = E == 8 ? 4 : GN_R;  // units of a lane at once
  const int lane = threadIdx.x & 63, groups = cdiv(a.slots, GN_NT / 64), per = groups * a.cchunks;
  const int n = blockIdx.x / per, rest = blockIdx.x - n * per, cc = rest % a.cchunks;
  const int slot = rest / a.cchunks * (GN_NT / 64) + (threadIdx.x >> 6);
  if (slot >= a.slots) return;
  const int u = lane & (a.cup - 1), rpp = 64 / a.cup, c = (cc * a.cu + u) * E;
  const long long r0 = (long long)slot * a.srows + lane / a.cup, r1 = min(a.HW, (slot + 1LL) * a.srows);
  const bool on = u < a.cu && c < a.C;
  const T* x = (const T*)a.x + n * a.HW * a.C + c;
  float cnt = 0.f, mean[E], m2[E];
#pragma unroll
  for (int e = 0; e < E; ++e) mean[e] = m2[e] = 0.f;
  for (long long r = r0; on && r < r1; r += (long long)S * rpp) {
    GnUnit<T, E> d[S];
    const int k = (int)min((long long)S, (r1 - r + rpp - 1) / rpp);
    float s[E], q[E], v[E];
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (i < k) d[i].load(x + (r + (long long)i * rpp) * a.C);
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = q[e] = 0.f;
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (i < k) {
        d[i].get(v);
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] += v[e];
      }
    const float inv = 1.f / k;
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] *= inv;
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (i < k) {
        gn_renew(d[i].u);
        d[i].get(v);
#pragma unroll
        for (int e = 0; e < E; ++e) q[e] += (v[e] - s[e]) * (v[e] - s[e]);
      }
    const float t = cnt + k, f = k / t, w = cnt * f;
    cnt = t;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = s[e] - mean[e];
      mean[e] += d * f;
      m2[e] += q[e] + d * d * w;
    }
  }
  for (int o = a.cup; o < 64; o <<= 1) {
    // both lanes of a pair get the same bits: the lower one's values come first
    const float other = __shfl_xor(cnt, o, 64);
    const bool upper = lane & o;
    const float n0 = upper ? other : cnt, n1 = upper ? cnt : other, t = n0 + n1;
    const float f = t > 0.f ? n1 / t : 0.f, w = n0 * f;
    cnt = t;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float om = __shfl_xor(mean[e], o, 64), oq = __shfl_xor(m2[e], o, 64);
      const float ma = upper ? om : mean[e], d = (upper ? mean[e] : om) - ma;
      mean[e] = ma + d * f;
      m2[e] += oq + d * d * w;
    }
  }
  if (on && lane < a.cup) {
    float* o = a.part + 2 * (((long long)n * a.slots + slot) * a.C + c);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      o[2 * e] = mean[e];
      o[2 * e + 1] = m2[e];
    }
  }
}

__device__ __forceinline__ float block_sum(float v, float* red) {  // red: 4 floats
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// mean and rstd of a (sample, group) from its slots' channels: a block each.
__global__ __launch_bounds__(GN_NT) void gn_mean_kernel(GnArgs a) {
  __shared__ float red[4];
  const int n = blockIdx.x / a.G, g = blockIdx.x - n * a.G;
  const float* part = a.part + 2 * ((long long)n * a.slots * a.C + g * a.gs);
  const int count = a.slots * a.gs;
  const float inv = 1.f / ((float)a.HW * a.gs);
  const float last = (float)(a.HW - (a.slots - 1LL) * a.srows);
  float s = 0.f;
  for (int i = threadIdx.x; i < count; i += GN_NT) {
    const int k = i / a.gs, c = i - k * a.gs;
    s += part[2 * ((long long)k * a.C + c)] * ((k == a.slots - 1 ? last : (float)a.srows) * inv);
  }
  const float mean = block_sum(s, red);
  float q = 0.f;
  for (int i = threadIdx.x; i < count; i += GN_NT) {
    const int k = i / a.gs, c = i - k * a.gs;
    const float* p = part + 2 * ((long long)k * a.C + c);
    q += p[1] + (k == a.slots - 1 ? last : (float)a.srows) * (p[0] - mean) * (p[0] - mean);
  }
  const float var = block_sum(q, red) * inv;
  if (threadIdx.x == 0) {
    a.mean[blockIdx.x] = mean;
    a.rstd[blockIdx.x] = 1.f / sqrtf(var + a.eps);
  }
}

// A thread's per-channel constants.
template <int E> struct GnChan {
  float mean[E], rstd[E], gamma[E], beta[E];
  __device__ __forceinline__ void load(const GnArgs& a, int n, int c) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int g = (c + e) / a.gs;
      mean[e] = a.mean[(long long)n * a.G + g];
      rstd[e] = a.rstd[(long long)n * a.G + g];
    }
    affine(a, c);
  }
  __device__ __forceinline__ void affine(const GnArgs& a, int c) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      gamma[e] = a.gamma ? a.gamma[c + e] : 1.f;
      beta[e] = a.beta ? a.beta[c + e] : 0.f;
    }
  }
  // Rounded after every operation, so that forward and backward (and whoever
  // follows the formula in fp32) see the same sign at a ReLU.
  __device__ __forceinline__ float xhat(int e, float x) const {
#pragma clang fp contract(off)
    return (x - mean[e]) * rstd[e];
  }
  __device__ __forceinline__ float pre(int e, float xh) const {
#pragma clang fp contract(off)
    return xh * gamma[e] + beta[e];
  }
};

template <typename T, int E, int ACT>
__global__ __launch_bounds__(GN_NT) void gn_apply_kernel(GnArgs a) {
  const GnPlace p = gn_place<E>(a);
  if (!p.on) return;
  GnChan<E> ch;
  ch.load(a, p.n, p.c);
  const long long base = p.n * a.HW * a.C + p.c;
  const T* x = (const T*)a.x + base;
  T* y = (T*)a.out + base;
  constexpr int A = 4;  // loads in flight
  for (long long r = p.r0 + p.r; r < p.r1; r += (long long)A * p.rpp) {
    GnUnit<T, E> u[A];
#pragma unroll
    for (int i = 0; i < A; ++i)
      if (r + i * p.rpp < p.r1) u[i].load(x + (r + i * p.rpp) * a.C);
#pragma unroll
    for (int i = 0; i < A; ++i)
      if (r + i * p.rpp < p.r1) {
        float v[E];
        u[i].get(v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = act_fwd<ACT, T>(ch.pre(e, ch.xhat(e, v[e])));
        GnUnit<T, E>::store(y + (r + i * p.rpp) * a.C, v);
      }
  }
}

// part[n][chunk][2][c] = sum g, and sum g * xhat, of the chunk's pixels.
template <typename T, int E, int ACT>
__global__ __launch_bounds__(GN_NT) void gn_bwd_sums_kernel(GnArgs a) {
  __shared__ float red[GN_NT * E];
  const GnPlace p = gn_place<E>(a);
  float s[E], q[E];
#pragma unroll
  for (int e = 0; e < E; ++e) s[e] = q[e] = 0.f;
  if (p.on) {
    GnChan<E> ch;
    ch.load(a, p.n, p.c);
    const long long base = p.n * a.HW * a.C + p.c;
    const T *x = (const T*)a.x + base, *dy = (const T*)a.dy + base;
    for (long long r = p.r0 + p.r; r < p.r1; r += p.rpp) {
      GnUnit<T, E> ux, ud;
      float v[E], d[E];
      ux.load(x + r * a.C);
      ud.load(dy + r * a.C);
      ux.get(v);
      ud.get(d);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = ch.xhat(e, v[e]), g = act_bwd<ACT, T>(d[e], ch.pre(e, xh));
        s[e] += g;
        q[e] += g * xh;
      }
    }
  }
  gn_row_sum<E>(s, red, a.cup);
  gn_row_sum<E>(q, red, a.cup);
  if (p.r == 0 && p.on) {
    float* o = a.part + 2 * ((long long)p.n * a.chunks + p.chunk) * a.C + p.c;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      o[e] = s[e];
      o[a.C + e] = q[e];
    }
  }
}

// Sums of src's columns over `per` rows a slice: 32 columns a block, 32 threads
// a column.  out: [slice][cols]; null: the sums are dbeta and dgamma.
struct GnColumns {
  const float* src;
  long long rows, per;
  int cols, blocks;  // blocks of a slice
  float* out;
};
__device__ __forceinline__ void gn_columns(const GnArgs& a, const GnColumns& k, int b) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, slice = b / k.blocks;
  const int c = (b - slice * k.blocks) * 32 + x;
  const long long r1 = min(k.rows, (slice + 1) * k.per);
  float s = 0.f;
  if (c < k.cols)
#pragma unroll 8
    for (long long r = slice * k.per + y; r < r1; r += 32) s += k.src[r * k.cols + c];
  red[y][x] = s;
  __syncthreads();
  for (int h = 16; h > 0; h >>= 1) {
    if (y < h) red[y][x] += red[y + h][x];
    __syncthreads();
  }
  if (y == 0 && c < k.cols) {
    if (k.out)
      k.out[(long long)slice * k.cols + c] = red[0][x];
    else
      (c < a.C ? a.dbeta + c : a.dgamma + (c - a.C))[0] = red[0][x];
  }
}
__global__ __launch_bounds__(1024) void gn_columns_kernel(GnArgs a, GnColumns k) { gn_columns(a, k, blockIdx.x); }

// Blocks from `first` on: coef = (avg h, avg h * xhat) of 4 (sample, group)s,
// 256 threads each, from the chunks' partial sums; those before: column sums.
__global__ __launch_bounds__(1024) void gn_bwd_coef_kernel(GnArgs a, GnColumns k, int first) {
  __shared__ float red[2][16];
  if ((int)blockIdx.x < first) {
    gn_columns(a, k, blockIdx.x);
    return;
  }
  const int t = threadIdx.x & 255, w = threadIdx.x >> 6;
  const long long i = ((long long)blockIdx.x - first) * 4 + (threadIdx.x >> 8);
  const int n = (int)(i / a.G), g = (int)(i - (long long)n * a.G);
  float s = 0.f, q = 0.f;
  if (n < a.N) {
    const float* part = a.part + (long long)n * a.chunks * 2 * a.C + g * a.gs;
    const int count = a.chunks * a.gs;
    for (int j = t; j < count; j += 256) {
      const int r = j / a.gs, c = j - r * a.gs;
      const float* p = part + (long long)r * 2 * a.C + c;
      const float m = a.gamma ? a.gamma[g * a.gs + c] : 1.f;
      s += m * p[0];
      q += m * p[a.C];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    q += __shfl_xor(q, o, 64);
  }
  if ((threadIdx.x & 63) == 0) {
    red[0][w] = s;
    red[1][w] = q;
  }
  __syncthreads();
  if (t == 0 && n < a.N) {
    const float inv = 1.f / ((float)a.HW * a.gs);
    a.coef[2 * i] = ((red[0][w] + red[0][w + 1]) + (red[0][w + 2] + red[0][w + 3])) * inv;
    a.coef[2 * i + 1] = ((red[1][w] + red[1][w + 1]) + (red[1][w + 2] + red[1][w + 3])) * inv;
  }
}

template <typename T, int E, int ACT>
__global__ __launch_bounds__(GN_NT) void gn_bwd_apply_kernel(GnArgs a) {
  const GnPlace p = gn_place<E>(a);
  if (!p.on) return;
  GnChan<E> ch;
  ch.load(a, p.n, p.c);
  float ca[E], cb[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float* k = a.coef + 2 * ((long long)p.n * a.G + (p.c + e) / a.gs);
    ca[e] = k[0];
    cb[e] = k[1];
  }
  const long long base = p.n * a.HW * a.C + p.c;
  const T *x = (const T*)a.x + base, *dy = (const T*)a.dy + base;
  T* dx = (T*)a.out + base;
  for (long long r = p.r0 + p.r; r < p.r1; r += p.rpp) {
    GnUnit<T, E> ux, ud;
    float v[E], d[E];
    ux.load(x + r * a.C);
    ud.load(dy + r * a.C);
    ux.get(v);
    ud.get(d);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float xh = ch.xhat(e, v[e]), h = act_bwd<ACT, T>(d[e], ch.pre(e, xh)) * ch.gamma[e];
      v[e] = ch.rstd[e] * (h - ca[e] - xh * cb[e]);
    }
    GnUnit<T, E>::store(dx + r * a.C, v);
  }
}

int next_pow2(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

// --------------------------------------------------------- one pass in all
// A block takes whole groups of one sample, U units a row, and keeps them in
// registers (up to R units a thread) from the sums to the results.  What runs
// once is bound by fetching its instructions (a kernel of 6000 took 14 us for
// one sample of 400 KB), so loops over registers end at the thread's units and
// everything else is kept short.
constexpr int GN_MOST = 1024;                          // threads of a block
constexpr int GN_WIDE = 256;                           // most units of a row
template <int E> constexpr int GN_SLOTS = 16 * 64 * E;  // floats: 16 waves of 64 units

struct GnFuse {
  int U, up, lup, W;  // units of a row, the next power of two, its logarithm, channels
  int rpp;            // rows of a pass
  int lanes;          // that add up a group
  int need;           // units of a thread
  int chunks;         // blocks of a sample
  int spread;         // samples go round the XCDs, so that blocks sharing cache lines share an L2
};

// A thread's place: its unit u of rows r, r + rpp, ..
template <typename T, int E> struct GnSeat {
  int n, c0, u, r;
  bool on, last;       // whether it has a unit at all, and one in the last pass
  uint32_t off, step;  // bytes from the sample's start, and from row to row
  __device__ __forceinline__ bool init(const GnArgs& a, const GnFuse& f) {
    const int b = blockIdx.x, k = f.spread ? b >> 3 : b;
    n = k / f.chunks;
    const int chunk = k - n * f.chunks;
    if (f.spread) n = (b & 7) + 8 * n;
    const int t = threadIdx.x;
    u = t & (f.up - 1);
    r = t >> f.lup;
    c0 = chunk * f.W;
    on = u < f.U;
    last = on && r + (f.need - 1) * f.rpp < (int)a.HW;
    off = ((uint32_t)r * a.C + c0 + u * E) * (uint32_t)sizeof(T);
    step = (uint32_t)f.rpp * a.C * (uint32_t)sizeof(T);
    return n < a.N;
  }
  // Pass i of f.need: whether this thread has a unit in it.
  __device__ __forceinline__ bool has(const GnFuse& f, int i) const { return i + 1 < f.need ? on : last; }
  __device__ __forceinline__ const T* at(const T* sample, int i) const {
    return (const T*)((const char*)sample + (off + i * step));
  }
  __device__ __forceinline__ T* at(T* sample, int i) const { return (T*)((char*)sample + (off + i * step)); }
};

// red[slot][c] = sums of the block's channels over the lanes of a wave (over
// one row, where a row is longer than a wave), all in a fixed order.
template <int E>
__device__ __forceinline__ void gn_lane_sums(const GnFuse& f, float (&v)[E], int u, bool on, float* red) {
  const int t = threadIdx.x;
  for (int o = f.up; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += __shfl_xor(v[e], o, 64);
  const int l = max(f.lup, 6);
  if (on && (t & ((1 << l) - 1)) < f.up)
#pragma unroll
    for (int e = 0; e < E; ++e) red[(t >> l) * f.W + u * E + e] = v[e];
}
// gsum[g] = the sum of a group's channels over the slots, times gamma where
// given: f.lanes lanes a group.
__device__ __forceinline__ void gn_group_sums(const GnArgs& a, const GnFuse& f, const float* red,
                                              const float* gamma, float* gsum) {
  const int t = threadIdx.x, L = f.lanes, slots = blockDim.x >> max(f.lup, 6), groups = f.W / a.gs;
  for (int g = t / L; g < groups; g += blockDim.x / L) {
    float s = 0.f;
    for (int c = g * a.gs + (t & (L - 1)); c < (g + 1) * a.gs; c += L) {
      float k = 0.f;
#pragma unroll 4
      for (int i = 0; i < slots; ++i) k += red[i * f.W + c];
      s += gamma ? k * gamma[c] : k;
    }
    for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    gsum[g] = s;
  }
}
// The sums of the groups of a unit's channels.
template <int E>
__device__ __forceinline__ void gn_spread(const GnArgs& a, const GnFuse& f, const float* gsum, int u, float (&out)[E]) {
  int g = u < f.U ? u * E / a.gs : 0, rest = u < f.U ? u * E - g * a.gs : 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    out[e] = gsum[g];
    const bool next = ++rest == a.gs;
    rest = next ? 0 : rest;
    g = next && e + 1 < E ? g + 1 : g;
  }
}

template <typename T, int E, int ACT, int R>
__global__ __launch_bounds__(GN_MOST) void gn_fused_kernel(GnArgs a, GnFuse f) {
  __shared__ float red[2][GN_SLOTS<E>], gsum[2][GN_WIDE * E];
  GnSeat<T, E> p;
  if (!p.init(a, f)) return;
  const T* x = (const T*)a.x + p.n * a.HW * a.C;
  T* y = (T*)a.out + p.n * a.HW * a.C;
  GnUnit<T, E> d[R];
  float s[E] = {}, v[E];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) d[i].load(p.at(x, i));
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      d[i].get(v);
#pragma unroll
      for (int e = 0; e < E; ++e) s[e] += v[e];
    }
  }
  const float inv = 1.f / ((float)a.HW * a.gs);
  GnChan<E> ch;
  gn_lane_sums(f, s, p.u, p.on, red[0]);
  __syncthreads();
  gn_group_sums(a, f, red[0], nullptr, gsum[0]);
  __syncthreads();
  gn_spread(a, f, gsum[0], p.u, ch.mean);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    ch.mean[e] *= inv;
    s[e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      gn_renew(d[i].u);
      d[i].get(v);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] -= ch.mean[e];
        s[e] += v[e] * v[e];
      }
    }
  }
  gn_lane_sums(f, s, p.u, p.on, red[1]);
  __syncthreads();
  gn_group_sums(a, f, red[1], nullptr, gsum[1]);
  __syncthreads();
  const long long g0 = (long long)p.n * a.G + p.c0 / a.gs;
  for (int g = threadIdx.x; g < f.W / a.gs; g += blockDim.x) {
    a.mean[g0 + g] = gsum[0][g] * inv;
    a.rstd[g0 + g] = 1.f / sqrtf(gsum[1][g] * inv + a.eps);
  }
  if (!p.on) return;
  gn_spread(a, f, gsum[1], p.u, ch.rstd);
#pragma unroll
  for (int e = 0; e < E; ++e) ch.rstd[e] = 1.f / sqrtf(ch.rstd[e] * inv + a.eps);
  ch.affine(a, p.c0 + p.u * E);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      gn_renew(d[i].u);
      d[i].get(v);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = act_fwd<ACT, T>(ch.pre(e, ch.xhat(e, v[e])));
      GnUnit<T, E>::store(p.at(y, i), v);
    }
  }
}

template <typename T, int E, int ACT, int R>
__global__ __launch_bounds__(GN_MOST) void gn_fused_bwd_kernel(GnArgs a, GnFuse f) {
  __shared__ float red[2][GN_SLOTS<E>], gsum[2][GN_WIDE * E];
  GnSeat<T, E> p;
  if (!p.init(a, f)) return;
  const T* x = (const T*)a.x + p.n * a.HW * a.C;
  const T* dy = (const T*)a.dy + p.n * a.HW * a.C;
  T* dx = (T*)a.out + p.n * a.HW * a.C;
  GnUnit<T, E> ux[R], uy[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      ux[i].load(p.at(x, i));
      uy[i].load(p.at(dy, i));
    }
  }
  GnChan<E> ch;
  if (p.on) ch.load(a, p.n, p.c0 + p.u * E);
  float s[E] = {}, q[E] = {}, v[E], w[E];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      ux[i].get(v);
      uy[i].get(w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = ch.xhat(e, v[e]), g = act_bwd<ACT, T>(w[e], ch.pre(e, xh));
        s[e] += g;
        q[e] += g * xh;
      }
    }
  }
  const float inv = 1.f / ((float)a.HW * a.gs), *gamma = a.gamma ? a.gamma + p.c0 : nullptr;
  gn_lane_sums(f, s, p.u, p.on, red[0]);
  gn_lane_sums(f, q, p.u, p.on, red[1]);
  __syncthreads();
  gn_group_sums(a, f, red[0], gamma, gsum[0]);
  gn_group_sums(a, f, red[1], gamma, gsum[1]);
  for (int c = threadIdx.x; c < 2 * f.W; c += blockDim.x) {  // the channels' totals
    const int w = c >= f.W, k = c - w * f.W, slots = blockDim.x >> max(f.lup, 6);
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < slots; ++i) sum += red[w][i * f.W + k];
    a.tot[((long long)p.n * 2 + w) * a.C + p.c0 + k] = sum;
  }
  __syncthreads();
  if (!p.on) return;
  gn_spread(a, f, gsum[0], p.u, s);
  gn_spread(a, f, gsum[1], p.u, q);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    s[e] *= inv;
    q[e] *= inv;
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (i < f.need && p.has(f, i)) {
      gn_renew(ux[i].u);
      gn_renew(uy[i].u);
      ux[i].get(v);
      uy[i].get(w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = ch.xhat(e, v[e]), h = act_bwd<ACT, T>(w[e], ch.pre(e, xh)) * ch.gamma[e];
        v[e] = ch.rstd[e] * (h - s[e] - xh * q[e]);
      }
      GnUnit<T, E>::store(p.at(dx, i), v);
    }
  }
}

// How a call is cut.  Chunks of pixels: 8 per thread at least, and no more
// than 1024 a sample, nor than give about 8 blocks per CU.
void gn_cut(GnArgs& a, int E) {
  const int units = a.C / E;
  a.cchunks = cdiv(units, 64);
  a.cu = cdiv(units, a.cchunks);
  a.cup = next_pow2(a.cu);
  const int rpp = GN_NT / a.cup;
  const long long blocks = (long long)a.N * a.cchunks;
  const long long want = std::min<long long>(1024, std::max<long long>(1, 2048 / std::max(1LL, blocks)));
  const long long least = (long long)GN_R * rpp;
  long long rows = std::max(least, cdivl(a.HW, want));
  rows = cdivl(rows, least) * least;
  a.rows = (int)std::min<long long>(rows, INT_MAX);
  a.chunks = (int)cdivl(a.HW, a.rows);
  // slots: 16 units a lane, no more than 512 a sample (a block reads those of a
  // group), nor than give 8192 waves
  const long long few = (long long)GN_R * 2 * (64 / a.cup);
  const long long most = std::min<long long>(512, std::max<long long>(4, 8192 / std::max(1LL, blocks)));
  a.srows = (int)std::min<long long>(cdivl(std::max(few, cdivl(a.HW, most)), few) * few, INT_MAX);
  a.slots = (int)cdivl(a.HW, a.srows);
}

bool unit_ok(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Calls `go` over the samples in groups whose grids stay below 2^21 blocks (2^31
// threads); `per` blocks a sample.
template <typename F> hipError_t gn_samples(GnArgs a, size_t esize, long long per, F&& go) {
  const long long most = std::max<long long>(8, (1 << 21) / per / 8 * 8), N = a.N;
  for (long long n = 0; n < N; n += most) {
    GnArgs b = a;
    b.N = (int)std::min(most, N - n);
    const size_t off = (size_t)n * a.HW * a.C * esize;
    b.x = (const char*)a.x + off;
    if (a.dy) b.dy = (const char*)a.dy + off;
    b.out = (char*)a.out + off;
    b.mean = a.mean + n * a.G;
    b.rstd = a.rstd + n * a.G;
    b.part = a.part + n * (a.dy ? a.chunks : a.slots) * 2 * a.C;
    if (a.tot) b.tot = a.tot + n * 2 * a.C;
    if (a.coef) b.coef = a.coef + n * 2 * a.G;
    EKYA_HIP(go(b, dim3((unsigned)(b.N * per))));
  }
  return hipSuccess;
}

// Threads and channels of the one-pass kernels, or false where a block cannot
// hold its groups: `most` units a thread.  Rows of a block are 128 bytes wide
// where that leaves 512 blocks.
bool gn_fuse(const GnArgs& a, int E, int bytes, int most, GnFuse& f, int& threads) {
  if (a.HW > GN_MOST * most || a.N > (1 << 20)) return false;
  const int base = a.gs / std::gcd(a.gs, E) * E, pieces = a.C / base;  // whole groups, whole units
  if (a.C % base) return false;
  auto fits = [&](int k) {
    const int up = next_pow2(base * k / E);
    return up <= GN_WIDE && a.HW <= (long long)GN_MOST / up * most;
  };
  int k = 1;
  for (int j = 2; j <= pieces && base * k * bytes < 128; ++j)
    if (pieces % j == 0 && fits(j) && (long long)a.N * (pieces / j) >= 512) k = j;
  if (!fits(k) || (k < pieces && base * k * bytes < 32 && (long long)a.N * a.HW * a.C > (1 << 20))) return false;
  f.W = base * k;
  f.U = f.W / E;
  f.up = next_pow2(f.U);
  f.chunks = a.C / f.W;
  f.spread = a.N >= 64 && f.chunks > 1;
  threads = 64;
  while (threads < GN_MOST && (threads * 2 < a.HW * f.up || threads < f.up)) threads *= 2;
  f.rpp = threads / f.up;
  f.need = (int)cdivl(a.HW, f.rpp);
  f.lup = 0;
  while (1 << f.lup < f.up) ++f.lup;
  f.lanes = 64;
  while (f.lanes > 1 && (f.lanes * (f.W / a.gs) > threads || f.lanes / 2 >= a.gs)) f.lanes /= 2;
  return f.need <= most;
}

template <typename T, int E, typename F>
hipError_t gn_fused_samples(const GnArgs& a, const GnFuse& f, F&& go) {
  return gn_samples(a, sizeof(T), f.chunks, [&](const GnArgs& b, dim3) {
    return go(b, dim3((unsigned)((f.spread ? (b.N + 7) / 8 * 8 : b.N) * f.chunks)));
  });
}

// Units of a thread: 64 of its 128 registers (1024 threads a block) hold them in
// fp32 and in the backward pass, whose units are pairs; bf16 forward stays at the
// same 16, with which two blocks fit a CU.  A call takes the smallest kernel that
// holds its units, since a short sample is bound by fetching code (128 x 784 x 128
// backward with 8 units 28.1 us, with 16 30.2; 4096 pixels of 64 channels with 16
// 37.4 forward and 68.4 backward, in several launches 49.3 and 76.1).
template <typename T, bool BACK> constexpr int GN_UNITS = BACK && sizeof(T) == 4 ? 8 : 16;
template <int MOST, typename F> auto gn_units(int need, F&& f) {
  if (need <= 3) return f(std::integral_constant<int, 3>{});
  if constexpr (MOST > 8)
    if (need > 8) return f(std::integral_constant<int, MOST>{});
  return f(std::integral_constant<int, 8>{});
}

template <typename T, int E> hipError_t gn_forward(GnArgs a, int act, hipStream_t st) {
  if constexpr (E > 1) {
    constexpr int EU = 4, R = GN_UNITS<T, false>;
    GnFuse f;
    int threads;
    if (gn_fuse(a, EU, sizeof(T), R, f, threads))
      return gn_fused_samples<T, EU>(a, f, [&](const GnArgs& b, dim3 grid) {
        return act_dispatch(act, [&](auto k) {
          return gn_units<R>(f.need, [&](auto r) {
            hipLaunchKernelGGL((gn_fused_kernel<T, EU, k.value, r.value>), grid, dim3(threads), 0, st, b, f);
            return hipGetLastError();
          });
        });
      });
  }
  gn_cut(a, E);
  const long long per = (long long)a.chunks * a.cchunks;
  EKYA_HIP(gn_samples(a, sizeof(T), cdivl(a.slots, GN_NT / 64) * a.cchunks, [&](const GnArgs& b, dim3 grid) {
    hipLaunchKernelGGL((gn_stats_kernel<T, E>), grid, dim3(GN_NT), 0, st, b);
    return hipGetLastError();
  }));
  EKYA_HIP(gn_samples(a, sizeof(T), a.G, [&](const GnArgs& b, dim3 grid) {
    hipLaunchKernelGGL(gn_mean_kernel, grid, dim3(GN_NT), 0, st, b);
    return hipGetLastError();
  }));
  return gn_samples(a, sizeof(T), per, [&](const GnArgs& b, dim3 grid) {
    return act_dispatch(act, [&](auto k) {
      hipLaunchKernelGGL((gn_apply_kernel<T, E, k.value>), grid, dim3(GN_NT), 0, st, b);
      return hipGetLastError();
    });
  });
}

// dbeta and dgamma as the column sums of src [rows][2 C]; more than GN_ROWS rows
// are first added up in slices, into a.slices.
constexpr long long GN_ROWS = 4096;
constexpr int GN_SLICES = 128;
hipError_t gn_param(const GnArgs& a, const float* src, long long rows, GnColumns& k, hipStream_t st) {
  k = {src, rows, std::max(1LL, rows), 2 * a.C, cdiv(2 * a.C, 32), nullptr};
  if (rows <= GN_ROWS) return hipSuccess;
  k.per = cdivl(rows, GN_SLICES);
  k.out = a.slices;
  const long long slices = cdivl(rows, k.per);
  hipLaunchKernelGGL(gn_columns_kernel, dim3((unsigned)(slices * k.blocks)), dim3(1024), 0, st, a, k);
  k = {a.slices, slices, slices, k.cols, k.blocks, nullptr};
  return hipGetLastError();
}

template <typename T, int E> hipError_t gn_backward(GnArgs a, int act, hipStream_t st) {
  if constexpr (E > 1) {
    // 8-byte units in bf16: a unit's constants and sums take half the registers
    constexpr int EU = 4, R = GN_UNITS<T, true>;
    GnFuse f;
    int threads;
    if (gn_fuse(a, EU, sizeof(T), R, f, threads)) {
      EKYA_HIP((gn_fused_samples<T, EU>(a, f, [&](const GnArgs& b, dim3 grid) {
        return act_dispatch(act, [&](auto k) {
          return gn_units<R>(f.need, [&](auto r) {
            hipLaunchKernelGGL((gn_fused_bwd_kernel<T, EU, k.value, r.value>), grid, dim3(threads), 0, st, b, f);
            return hipGetLastError();
          });
        });
      })));
      if (!a.dgamma) return hipSuccess;
      GnColumns k;
      EKYA_HIP(gn_param(a, a.tot, a.N, k, st));
      hipLaunchKernelGGL(gn_columns_kernel, dim3(k.blocks), dim3(1024), 0, st, a, k);
      return hipGetLastError();
    }
  }
  gn_cut(a, E);
  const long long per = (long long)a.chunks * a.cchunks;
  EKYA_HIP(gn_samples(a, sizeof(T), per, [&](const GnArgs& b, dim3 grid) {
    return act_dispatch(act, [&](auto k) {
      hipLaunchKernelGGL((gn_bwd_sums_kernel<T, E, k.value>), grid, dim3(GN_NT), 0, st, b);
      return hipGetLastError();
    });
  }));
  GnColumns k{};
  if (a.dgamma) EKYA_HIP(gn_param(a, a.part, (long long)a.N * a.chunks, k, st));
  int first = k.blocks;  // the first launch takes the parameters' sums with it
  if (a.N == 0 && first) {
    hipLaunchKernelGGL(gn_columns_kernel, dim3(first), dim3(1024), 0, st, a, k);
    EKYA_HIP(hipGetLastError());
  }
  EKYA_HIP(gn_samples(a, sizeof(T), a.G, [&](const GnArgs& b, dim3) {
    hipLaunchKernelGGL(gn_bwd_coef_kernel, dim3((unsigned)(first + cdivl((long long)b.N * b.G, 4))), dim3(1024), 0,
                       st, b, k, first);
    first = 0;
    return hipGetLastError();
  }));
  return gn_samples(a, sizeof(T), per, [&](const GnArgs& b, dim3 grid) {
    return act_dispatch(act, [&](auto k) {
      hipLaunchKernelGGL((gn_bwd_apply_kernel<T, E, k.value>), grid, dim3(GN_NT), 0, st, b);
      return hipGetLastError();
    });
  });
}

GnArgs gn_args(int N, long long HW, int C, int G) {
  GnArgs a{};
  a.N = N;
  a.HW = HW;
  a.C = C;
  a.G = G;
  a.gs = C / G;
  return a;
}

size_t gn_part_floats(GnArgs a, int E) {
  gn_cut(a, E);
  return (size_t)a.N * std::max(a.chunks, a.slots) * 2 * a.C;
}

}  // namespace

// Scratch in floats, for either unit (addresses decide which one a call takes).
size_t groupnorm_workspace_floats(int dt, int N, long long HW, int C, int G, bool backward) {
  const GnArgs a = gn_args(N, HW, C, G);
  const int E = dtype_vec(dt);
  size_t f = gn_part_floats(a, 1);
  if (C % E == 0) f = std::max(f, gn_part_floats(a, E));
  if (backward) f += (size_t)N * 2 * (C + (size_t)G) + (size_t)GN_SLICES * 2 * C;
  return f;
}

hipError_t groupnorm_fwd(int dt, const void* x, int N, long long HW, int C, int G,
                         const float* gamma, const float* beta, float eps, int act, void* y,
                         float* mean, float* rstd, float* ws, hipStream_t st) {
  GnArgs a = gn_args(N, HW, C, G);
  a.x = x;
  a.out = y;
  a.gamma = gamma;
  a.beta = beta;
  a.eps = eps;
  a.mean = mean;
  a.rstd = rstd;
  a.part = ws;
  const bool unit = C % dtype_vec(dt) == 0 && unit_ok(x) && unit_ok(y);
  if (dt == DT_BF16)
    return unit ? gn_forward<bf16, 8>(a, act, st) : gn_forward<bf16, 1>(a, act, st);
  return unit ? gn_forward<float, 4>(a, act, st) : gn_forward<float, 1>(a, act, st);
}

hipError_t groupnorm_bwd(int dt, const void* dy, const void* x, int N, long long HW, int C, int G,
                         const float* gamma, const float* beta, const float* mean,
                         const float* rstd, int act, void* dx, float* dgamma, float* dbeta,
                         float* ws, hipStream_t st) {
  GnArgs a = gn_args(N, HW, C, G);
  a.x = x;
  a.dy = dy;
  a.out = dx;
  a.gamma = gamma;
  a.beta = beta;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.tot = ws;
  a.coef = a.tot + (size_t)N * 2 * C;
  a.slices = a.coef + (size_t)N * 2 * G;
  a.part = a.slices + (size_t)GN_SLICES * 2 * C;
  const bool unit = C % dtype_vec(dt) == 0 && unit_ok(x) && unit_ok(dy) && unit_ok(dx);
  if (dt == DT_BF16)
    return unit ? gn_backward<bf16, 8>(a, act, st) : gn_backward<bf16, 1>(a, act, st);
  return unit ? gn_backward<float, 4>(a, act, st) : gn_backward<float, 1>(a, act, st);
}

}  // namespace ekya
