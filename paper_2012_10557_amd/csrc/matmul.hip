// Matrix products with everything elementwise behind them in the same kernel,
// and their gradients.
//
//   D[r][c] = sum_t A(r, t) B(c, t)
//
//   forward  y[m][n]:  A = w[n][k],  B = x[m][k],   t = k
//   dx[m][k]:          A = w[n][k]^, B = dz[m][n],  t = n
//   dw[n][k]:          A = x[m][k]^, B = dz[m][n]^, t = m
//
// r is the direction in which the result lies in memory, t the reduction; an
// operand marked ^ lies in memory with t as its rows.  A block of 4 or 8 waves
// owns a tile of D; stages of 128 bytes of the reduction per row (64 bf16, 32
// fp32: whole cache lines) pass through two or three buffers in LDS, and the fragments
// of the next half stage are read into registers while the matrix cores work on
// this one's.
//
// Long products are bound by the matrix cores and how steadily they are fed
// (8192^3 bf16 1340 TFLOP/s, 820 us, where the vendor's library takes 664; fp32 4096
// x 2048 x 2048 140 of the library's 146 TFLOP/s), short ones by what a tile costs besides its
// stages: launch, the first loads, and the epilogue, which overlaps with nothing
// where a CU holds one block (16384 x 2048 x 8192 with SiLU and a residual 519 us,
// 469 without both).
#include <algorithm>

#include "act.hpp"
#include "kernels.hpp"
#include "matmul_plan.hpp"

namespace ekya {
namespace {

__device__ __align__(16) uint4 g_mm_zero[1];

// The wave's own LDS accesses are done, then all waves meet; what waves still
// have in flight from global memory is left in flight.
__device__ __forceinline__ void mm_wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void mm_barrier() {
  mm_wait_lds();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <typename T> struct MmArgs {
  const T *a, *b;
  long long lda, ldb;
  long long R, C, Tn;  // outputs along r and c, reduction length
  long long Ra, Cb;    // outputs that a and b hold in memory (more than R and C in a padded copy)
  const float* bias;   // [R] or null
  const T* res;        // [C][R] or null
  long long ldr;
  int res_first;
  void* y;  // [C][R]
  long long ldy;
  T* z;     // [C][R] or null
  long long ldz;
  int vec;      // bias, res, y and z allow 16-byte accesses at multiples of 16 outputs
  float* part;  // [split][C][Rp] where splits > 1
  long long Rp; // R up to a multiple of 4
  int tiles_r, tiles_c, splits, stages;  // stages of a split
};

// ------------------------------------------------------------- epilogue
// N elements by 16-byte accesses (8-byte ones for four bf16).
template <typename T, int N> __device__ __forceinline__ void load_run(const T* p, float (&v)[N]) {
  if constexpr (N < Elt<T>::E) return load4(p, v);
#pragma unroll
  for (int i = 0; i + Elt<T>::E <= N; i += Elt<T>::E) {
    Unit<T> t;
    t.u = *reinterpret_cast<const uint4*>(p + i);
#pragma unroll
    for (int e = 0; e < Elt<T>::E; ++e) v[i + e] = to_f(t.e[e]);
  }
}
template <typename T, int N> __device__ __forceinline__ void store_run(T* p, const float (&v)[N]) {
  if constexpr (N < Elt<T>::E) return store4(p, v);
#pragma unroll
  for (int i = 0; i + Elt<T>::E <= N; i += Elt<T>::E) {
    Unit<T> t;
#pragma unroll
    for (int e = 0; e < Elt<T>::E; ++e) t.e[e] = from_f<T>(v[i + e]);
    *reinterpret_cast<uint4*>(p + i) = t.u;
  }
}

// Finishes N outputs (r .. r + N - 1, c) by 16-byte accesses; v: the sums,
// bias and res: their N values (res: where there is one).
template <typename T, typename OT, int ACT, int N>
__device__ __forceinline__ void mm_finish(const MmArgs<T>& a, long long r, long long c, float (&v)[N],
                                          const float (&bias)[N], const float (&res)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] += bias[i];
  if (a.res_first)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += res[i];
  if (a.z) store_run(a.z + c * a.ldz + r, v);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = act_fwd<ACT, T>(v[i]);
  if (a.res && !a.res_first)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += res[i];
  store_run((OT*)a.y + c * a.ldy + r, v);
}
template <typename T, int N>
__device__ __forceinline__ void mm_bias(const MmArgs<T>& a, long long r, float (&bias)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = 0.f;
  if (a.bias) load_run(a.bias + r, bias);
}
// One output; bias and res: what is added (0 where there is none).
template <typename T, typename OT, int ACT>
__device__ __forceinline__ void mm_finish_one(const MmArgs<T>& a, long long r, long long c, float s, float bias,
                                              float res) {
  s += bias;
  if (a.res_first) s += res;
  if (a.z) a.z[c * a.ldz + r] = from_f<T>(s);
  s = act_fwd<ACT, T>(s);
  if (!a.res_first) s += res;
  ((OT*)a.y)[c * a.ldy + r] = from_f<OT>(s);
}

// ------------------------------------------------------------- operands
typedef short mm_v4i16 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 mm_read_tr(const char* p) {
  mm_v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) mm_v4i16*)(__attribute__((address_space(3))) char*)p);
  return __builtin_bit_cast(uint2, v);
}

// LDS layout of a stage.  Rows of t-contiguous operands are 8 units of 16
// bytes; unit u of row r is stored at u ^ f(r).  Operands with t as rows keep
// their rows of BX outputs; unit u of row t is stored at u ^ h(t).  f and h
// spread what 8 (16-byte reads) or 32 (8-byte reads) consecutive lanes touch
// over all 64 banks.
template <typename T, int BX, bool OC> struct MmOperand {
  static constexpr int E = Elt<T>::E;
  static constexpr int TS = 8 * E;               // reduction elements of a stage
  static constexpr int UNITS = BX * 8;           // units of a stage
  static constexpr int RU = OC ? BX / E : 8;     // units of a row in LDS
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (!OC) return row & 7;
    if constexpr (sizeof(T) == 4) return ((row >> 2) & 3) << 2;
    // 32 lanes read 32 bytes of each of rows 0 .. 3 and 8 .. 11 (and 16 on)
    if constexpr (BX == 64) return ((row >> 1) & 1) << 2 | ((row >> 3) & 1) << 1;  // rows of 128 bytes
    return (row & 3) << 1 | ((row >> 3) & 1) << 3;
  }
  // Where the unit stored at position q of a stage comes from: output x (of
  // the tile) and reduction element t (of the stage).
  static __device__ __forceinline__ void place(int q, int& x, int& t) {
    const int row = q / RU, u = (q % RU) ^ swizzle(row);
    x = OC ? u * E : row;
    t = OC ? row : u * E;
  }
  // Fragments of the wave whose outputs start at `x`, a multiple of 16, within
  // the tile: lane f of 16 holds output 16 i + f.
  // half: of the stage.
  template <int TF>
  static __device__ __forceinline__ void read(const uint4* s, int half, int x, int lane, uint4 (&f)[TF]) {
    const int fr = lane & 15, q = lane >> 4;
    if constexpr (!OC) {
      const uint4* p = s + (x + fr) * 8 + ((4 * half + q) ^ swizzle(fr));
#pragma unroll
      for (int i = 0; i < TF; ++i) f[i] = p[16 * i * 8];
    } else if constexpr (sizeof(T) == 2) {
      // lane 4 a + m of 16 supplies outputs 4 m .. 4 m + 3 of row a of four
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int t = half * 32 + q * 8 + k * 4 + (fr >> 2);
#pragma unroll
        for (int i = 0; i < TF; ++i) {
          const int o = x + 16 * i + 4 * (fr & 3);
          const char* p = (const char*)(s + t * RU + ((o / 8) ^ swizzle(t))) + (o & 4) * 2;
          const uint2 v = mm_read_tr(p);
          if (k == 0) { f[i].x = v.x; f[i].y = v.y; } else { f[i].z = v.x; f[i].w = v.y; }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < TF; ++i) {
        const int o = x + 16 * i + fr;
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = half * 16 + q * 4 + e;
          v[e] = reinterpret_cast<const uint32_t*>(s + t * RU + ((o / 4) ^ swizzle(t)))[o & 3];
        }
        f[i] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  }
};

// A unit from an address that may lie on any element.
template <typename T> __device__ __forceinline__ uint4 load_any(const T* p, int cnt) {
  Unit<T> t;
  t.u = zero_unit();
  if (cnt == Elt<T>::E) {
    __builtin_memcpy(&t.u, p, 16);
  } else {
#pragma unroll
    for (int e = 0; e < Elt<T>::E; ++e)
      if (e < cnt) t.e[e] = p[e];
  }
  return t.u;
}

// Workgroups go round the 8 XCDs; each XCD gets a contiguous range of (split,
// tile) items, whole splits where there are some (their tiles read the same
// part of both operands), and a range walks the tiles four rows at a time, so
// that the blocks an XCD runs together share panels of both operands in its L2.
__device__ __forceinline__ void mm_item(int L, int tiles_r, int tiles_c, int splits, int& split, int& tr, int& tc) {
  const int tiles = tiles_r * tiles_c, total = tiles * splits;
  const int x = L & 7, k = L >> 3;
  const int item = x * (total >> 3) + min(x, total & 7) + k;
  split = item / tiles;
  const int t = item - split * tiles;
  const int band = t / (4 * tiles_c), rest = t - band * 4 * tiles_c;
  const int h = min(4, tiles_r - 4 * band);
  tc = rest / h;
  tr = 4 * band + rest - tc * h;
}

// BR x BC tile, WR x WC waves, KG groups of them with a part of the reduction
// each (buffers of their own, sums added up at the end).  DMA: both operands are read in whole units on
// 16 bytes (global memory to LDS directly); else through registers.
template <typename T, typename OT, int BR, int BC, int WR, int WC, int NST, int KG, bool AOC, bool BOC, bool DMA, int ACT>
__global__ __launch_bounds__(WR* WC* KG * 64, 2) void mm_kernel(MmArgs<T> a) {
  constexpr int NW = WR * WC;
  constexpr int TI = BR / WR / 16, TJ = BC / WC / 16;
  static_assert(TI % 4 == 0, "64 outputs of A at a time");
  using OpA = MmOperand<T, BR, AOC>;
  using OpB = MmOperand<T, BC, BOC>;
  constexpr int TS = OpA::TS, SU = OpA::UNITS + OpB::UNITS;
  constexpr int LPS = SU / 64 / NW;  // units of a lane in a stage
  static_assert(OpA::UNITS % 64 == 0 && SU % (64 * NW) == 0, "whole copies");
  __shared__ uint4 buffers[KG * NST * SU];

  const int lane = threadIdx.x & 63;
  const int group = KG > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * NW;
  uint4* const smem = buffers + group * NST * SU;
  int split, tr, tc;
  mm_item(blockIdx.x, a.tiles_r, a.tiles_c, a.splits, split, tr, tc);
  const long long r0 = (long long)tr * BR, c0 = (long long)tc * BC;
  const long long part_t = (long long)a.stages * TS;  // reduction elements of a group
  const long long t_first = split * KG * part_t;      // the block's
  const long long t_begin = min(a.Tn, t_first + group * part_t), t_end = min(a.Tn, t_begin + part_t);
  const int ns = (int)cdivl(t_end - t_begin, TS);
  // all groups meet at the barriers of the first, which has the most stages
  const int most = KG > 1 ? (int)cdivl(min(a.Tn, t_first + part_t) - t_first, TS) : ns;

  // This lane's sources of the next stage.  Outputs past the end read what the
  // last one reads: their results are not stored.
  const T* src[LPS];
  int whole[LPS];  // without DMA: elements of the unit that exist within its row of outputs
#pragma unroll
  for (int j = 0; j < LPS; ++j) {
    const int q = (wave + NW * j) * 64;
    int x, u;
    if (q < OpA::UNITS) {
      OpA::place(q + lane, x, u);
      const long long last = AOC && DMA ? a.Ra - OpA::E : a.R - 1;
      const long long g = min(r0 + x, last), k = t_begin + u;
      src[j] = AOC ? a.a + k * a.lda + g : a.a + g * a.lda + k;
      whole[j] = AOC ? (int)min((long long)OpA::E, a.R - g) : OpA::E;
    } else {
      OpB::place(q - OpA::UNITS + lane, x, u);
      const long long last = BOC && DMA ? a.Cb - OpB::E : a.C - 1;
      const long long g = min(c0 + x, last), k = t_begin + u;
      src[j] = BOC ? a.b + k * a.ldb + g : a.b + g * a.ldb + k;
      whole[j] = BOC ? (int)min((long long)OpB::E, a.C - g) : OpB::E;
    }
  }
  const long long step_a = AOC ? TS * a.lda : TS, step_b = BOC ? TS * a.ldb : TS;
  // reduction elements of copy j's unit that exist when `left` remain at the
  // stage's start
  auto there = [&](int j, int left) {
    const int q = (wave + NW * j) * 64;
    int x, u;
    if (q < OpA::UNITS) {
      OpA::place(q + lane, x, u);
      return AOC ? (u < left ? whole[j] : 0) : max(0, min(OpA::E, left - u));
    }
    OpB::place(q - OpA::UNITS + lane, x, u);
    return BOC ? (u < left ? whole[j] : 0) : max(0, min(OpB::E, left - u));
  };
  const void* zero = g_mm_zero;
  asm volatile("" : "+s"(zero));
  auto left_at = [&](int s) { return (int)min((long long)TS, t_end - t_begin - (long long)s * TS); };
  auto copy_full = [&](int s) {  // DMA
    uint4* slot = smem + (s % NST) * SU;
#pragma unroll
    for (int j = 0; j < LPS; ++j) {
      dma16(src[j], slot + (wave + NW * j) * 64);
      src[j] += (wave + NW * j) * 64 < OpA::UNITS ? step_a : step_b;
    }
  };
  auto copy = [&](int s) {
    const int left = left_at(s);
    if (left == TS) return copy_full(s);
    uint4* slot = smem + (s % NST) * SU;  // the last stage
#pragma unroll
    for (int j = 0; j < LPS; ++j)
      dma16(there(j, left) ? (const void*)src[j] : zero, slot + (wave + NW * j) * 64);
  };
  constexpr int H = BR == 64 ? 2 : 1;  // without DMA: stages on their way in registers
  uint4 held[H][LPS];
  auto fetch = [&](int s, uint4 (&held)[LPS]) {
    const int left = left_at(s);
#pragma unroll
    for (int j = 0; j < LPS; ++j) {
      held[j] = load_any(src[j], left == TS ? whole[j] : there(j, left));
      src[j] += (wave + NW * j) * 64 < OpA::UNITS ? step_a : step_b;
    }
  };
  auto put = [&](int s, uint4 (&held)[LPS]) {
    uint4* slot = smem + (s % NST) * SU;
#pragma unroll
    for (int j = 0; j < LPS; ++j) slot[(wave + NW * j) * 64 + lane] = held[j];
  };

  const int xr = wave / WC * (BR / WR), xc = wave % WC * (BC / WC);
  uint4 fa[2][TI], fb[2][TJ];
  auto frags = [&](int s, int half) {
    const uint4* slot = smem + (s % NST) * SU;
    OpA::template read<TI>(slot, half, xr, lane, fa[half]);
    OpB::template read<TJ>(slot + OpA::UNITS, half, xc, lane, fb[half]);
  };

  f32x4 acc[TI][TJ];
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // A stage: read its second half and multiply the first; then the barrier ends
  // every wave's reads of it (its fragments are in registers), makes the next
  // one visible and frees its buffer; read the next one's first half and
  // multiply the second.
  if constexpr (DMA) {
#pragma unroll
    for (int p = 0; p < NST; ++p)
      if (p < ns) copy(p);
    if (ns >= NST) wait_vmcnt<LPS*(NST - 1)>(); else wait_vmcnt<0>();
  } else {
    fetch(0, held[0]);
    put(0, held[0]);
    if (ns > 1) {
      fetch(1, held[0]);
      put(1, held[0]);
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (2 + h < ns) fetch(2 + h, held[h]);
  }
  mm_barrier();
  frags(0, 0);
  int s = 0;
  if constexpr (DMA) {  // without a branch while whole stages follow
    int full = (int)((t_end - t_begin) / TS);  // of the last group, which has the fewest
    if constexpr (KG > 1) {
      const long long l = min(a.Tn, t_first + (KG - 1) * part_t);
      full = (int)((min(a.Tn, l + part_t) - l) / TS);
    }
    for (; s + NST < full; ++s) {
      frags(s, 1);
      mma_tile(acc, fa[0], fb[0], (T*)nullptr);
      wait_vmcnt<LPS*(NST - 2)>();
      mm_barrier();
      copy_full(s);
      frags(s + 1, 0);
      mma_tile(acc, fa[1], fb[1], (T*)nullptr);
    }
  }
  auto step = [&](int s, uint4 (&held)[LPS]) {
    const bool any = KG == 1 || s < ns;
    if (any) {
      frags(s, 1);
      mma_tile(acc, fa[0], fb[0], (T*)nullptr);
    }
    if constexpr (DMA) {
      if (s + NST - 1 < ns) wait_vmcnt<LPS*(NST - 2)>(); else wait_vmcnt<0>();
    }
    mm_barrier();
    if constexpr (DMA) {
      if (s + NST < ns) copy(s + NST);
    } else {
      if (s + 2 < ns) put(s + 2, held);
      if (s + 2 + H < ns) fetch(s + 2 + H, held);
    }
    if (any) {
      frags(s + 1, 0);  // after the last stage: not used
      mma_tile(acc, fa[1], fb[1], (T*)nullptr);
    }
  };
  for (; s < most; s += H) {
    step(s, held[0]);
    if constexpr (H == 2)
      if (s + 1 < ns) step(s + 1, held[1]);
  }
  if constexpr (KG > 1) {  // the first group adds the others' sums in their order
    static_assert(DMA && NW * TI * TJ * 64 <= NST * SU, "a group's sums fit its buffers");
    f32x4* sums = reinterpret_cast<f32x4*>(smem) + wave * TI * TJ * 64 + lane;
    mm_barrier();
    if (group > 0)
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) sums[(i * TJ + j) * 64] = acc[i][j];
    mm_barrier();
    if (group > 0) return;
    for (int g = 1; g < KG; ++g)
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] += sums[g * NST * SU + (i * TJ + j) * 64];
  }

  // 64 rows of the wave's tile at a time pass through its own part of LDS (no
  // wave reads stages any more), so that a lane finishes consecutive outputs in
  // a loop.  Without it, straight from the accumulators, the code was 10 times
  // as long and its fetching took most of a short reduction's time (6272 x 2048
  // x 512 with GELU: 54 us).
  const int fr = lane & 15, q = lane >> 4;
  const long long cw = c0 + xc;
  const int cols = (int)min((long long)TJ * 16, a.C - cw);
  float* part = a.part + split * a.C * a.Rp;
  f32x4* own = reinterpret_cast<f32x4*>(smem) + wave * 16 * TJ * 16;
  static_assert(NW * TJ * 16 * 64 * 4 <= NST * SU * 16, "64 rows of every wave");
#pragma unroll
  for (int g = 0; g < TI / 4; ++g) {
    mm_wait_lds();  // the wave's own accesses, in order
#pragma unroll
    for (int j = 0; j < TJ; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) own[(16 * j + fr) * 16 + ((4 * i + q) ^ fr)] = acc[4 * g + i][j];
    mm_wait_lds();  // the wave's own accesses, in order
    const long long r0w = r0 + xr + 64 * g;
    if (a.vec || a.splits > 1) {
      constexpr int N = 16 / sizeof(OT), L = 64 / N;  // outputs of a lane, lanes of a column
      constexpr int P = 64 / L, U = TJ * 16 / P < 8 ? TJ * 16 / P : 8;  // columns at once, steps in flight
      const long long r = r0w + lane % L * N;
      if (r + N <= a.R) {
        float bias[N];
        if (a.splits == 1) mm_bias(a, r, bias);
        const bool res = a.res && a.splits == 1;
        for (int k0 = lane / L; k0 < cols; k0 += P * U) {
          // the residual of all steps is on its way before the first is needed (of
          // four, 16384 x 2048 x 8192 with SiLU took 595 us, of eight 567)
          float w[U][N];
          if (res)
#pragma unroll
            for (int u = 0; u < U; ++u) load_run(a.res + (cw + min(k0 + u * P, cols - 1)) * a.ldr + r, w[u]);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = k0 + u * P;
            if (k >= cols) break;
            float v[N];
#pragma unroll
            for (int i = 0; i < N; i += 4) {
              const f32x4 x = own[k * 16 + ((lane % L * N + i) / 4 ^ (k & 15))];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[i + e] = x[e];
            }
            if (a.splits > 1)
              store_run(part + (cw + k) * a.Rp + r, v);
            else
              mm_finish<T, OT, ACT, N>(a, r, cw + k, v, bias, w[u]);
          }
        }
      }
    }
    // rows that do not fill a lane's outputs, or all of them where accesses of
    // 16 bytes are not possible: a lane takes one row
    const long long r = r0w + lane, first = a.vec || a.splits > 1 ? a.R / (16 / (int)sizeof(OT)) * (16 / (int)sizeof(OT)) : 0;
    if (r < a.R && r >= first) {
      const float bias = a.bias && a.splits == 1 ? a.bias[r] : 0.f;
      const T* res = a.res && a.splits == 1 ? a.res + cw * a.ldr + r : nullptr;
      // columns at once, whose residuals are on their way before the first is
      // needed (one after the other, 2000 x 333 x 2001 bf16 with SiLU and z took 46
      // us, 35 so; fp32 1001 x 513 x 771 23.8 and 20.5).  Eight times GELU is more
      // code than its fetching is worth: 333 x 211 x 777 10.0 us, 9.8 with four.
      constexpr int U = ACT == ACT_GELU ? 4 : 8;
#pragma unroll 1
      for (int k0 = 0; k0 < cols; k0 += U) {
        T w[U];
        if (res)
#pragma unroll
          for (int u = 0; u < U; ++u) w[u] = res[min(k0 + u, cols - 1) * a.ldr];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = k0 + u;
          if (k >= cols) break;
          const float v = reinterpret_cast<const float*>(own)[(k * 16 + ((lane >> 2) ^ (k & 15))) * 4 + (lane & 3)];
          if (a.splits > 1)
            part[(cw + k) * a.Rp + r] = v;
          else
            mm_finish_one<T, OT, ACT>(a, r, cw + k, v, bias, res ? to_f(w[u]) : 0.f);
        }
      }
    }
  }
}

// Adds up the splits in their order; N outputs a thread (1: accesses of 16
// bytes are not possible).
template <typename T, typename OT, int ACT, int N>
__global__ __launch_bounds__(256) void mm_reduce_kernel(MmArgs<T> a) {
  const long long per = cdivl(a.R, N), i = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long c = i / per, r = (i - c * per) * N, step = a.C * a.Rp;
  if (c >= a.C) return;
  const float* p = a.part + c * a.Rp + r;
  if constexpr (N > 1) if (r + N <= a.R) {
    float v[N] = {};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      float w[N];
      load_run(p + s * step, w);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] += w[e];
    }
    float bias[N], res[N];
    mm_bias(a, r, bias);
    if (a.res) load_run(a.res + c * a.ldr + r, res);
    mm_finish<T, OT, ACT, N>(a, r, c, v, bias, res);
    return;
  }
  for (int e = 0; e < N && r + e < a.R; ++e) {
    float v = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) v += p[s * step + e];
    mm_finish_one<T, OT, ACT>(a, r + e, c, v, a.bias ? a.bias[r + e] : 0.f,
                              a.res ? to_f(a.res[c * a.ldr + r + e]) : 0.f);
  }
}

// ---------------------------------------------------------------- host side
bool unit16(const void* p, long long ld, int dt) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % dtype_vec(dt) == 0;
}

long long round4(long long n) { return (n + 3) & ~3LL; }
size_t mm_part_floats(long long R, long long C, long long Tn, int dt, bool dma) {
  const MmPlan p = mm_plan(R, C, Tn, dt == DT_F32, dma);
  return p.splits > 1 ? (size_t)p.splits * C * round4(R) : 0;
}

constexpr long long MM_TILES = 1 << 21;  // tiles of a launch

template <typename T, typename OT, bool AOC, bool BOC, int ACT>
hipError_t mm_run(MmArgs<T> a, bool dma, hipStream_t st) {
  const MmPlan p = mm_plan(a.R, a.C, a.Tn, sizeof(T) == 4, dma);
  a.splits = p.splits;
  a.Rp = round4(a.R);
  a.stages = p.stages;
  // launches of at most MM_TILES tiles; a split product has few and goes in one
  const long long C = a.C, tiles_r = cdivl(a.R, p.tile);
  const long long cs = std::max(1LL, MM_TILES / tiles_r) * p.tile;
  for (long long c = 0; c < C; c += cs) {
    MmArgs<T> b = a;
    b.C = std::min(cs, C - c);
    b.b = a.b + (BOC ? c : c * a.ldb);
    b.Cb = a.Cb - c;
    if (a.res) b.res = a.res + c * a.ldr;
    if (a.z) b.z = a.z + c * a.ldz;
    b.y = (OT*)a.y + c * a.ldy;
    b.tiles_r = (int)tiles_r;
    b.tiles_c = (int)cdivl(b.C, p.tile);
    const dim3 grid((unsigned)((long long)b.tiles_r * b.tiles_c * b.splits));
    auto go = [&](auto tile, auto wr, auto wc, auto nst, auto kg, auto direct) {
      hipLaunchKernelGGL((mm_kernel<T, OT, tile.value, tile.value, wr.value, wc.value, nst.value, kg.value, AOC,
                                    BOC, direct.value, ACT>),
                         grid, dim3(wr.value * wc.value * kg.value * 64), 0, st, b);
    };
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    using I4 = std::integral_constant<int, 4>;
    using T64 = std::integral_constant<int, 64>;
    using T128 = std::integral_constant<int, 128>;
    using T256 = std::integral_constant<int, 256>;
    if constexpr (sizeof(T) == 2)
      if (p.tile == 256) go(T256{}, I2{}, I4{}, I2{}, I1{}, std::true_type{});
    if constexpr (sizeof(T) == 2)
      if (p.tile == 128 && p.groups == 2) go(T128{}, I2{}, I2{}, I2{}, I2{}, std::true_type{});
    if (p.tile == 128 && p.groups == 1 && dma) go(T128{}, I2{}, I2{}, I2{}, I1{}, std::true_type{});
    if (p.tile == 128 && !dma) go(T128{}, I2{}, I2{}, I2{}, I1{}, std::false_type{});
    // a CU's only block keeps three stages in flight (128 x 2048 x 8192: 18.6 us
    // with two, 12.6 with three); where it has more, two buffers leave them room
    // (1024 x 4096 x 512 with 512 tiles: 13.0 and 14.1 us)
    if (p.tile == 64 && dma && grid.x <= 256) go(T64{}, I1{}, I4{}, I3{}, I1{}, std::true_type{});
    if (p.tile == 64 && dma && grid.x > 256) go(T64{}, I1{}, I4{}, I2{}, I1{}, std::true_type{});
    if (p.tile == 64 && !dma) go(T64{}, I1{}, I4{}, I2{}, I1{}, std::false_type{});
    EKYA_HIP(hipGetLastError());
  }
  if (a.splits > 1) {
    const long long threads = a.C * cdivl(a.R, a.vec ? 16 / sizeof(T) : 1);
    const dim3 grid((unsigned)cdivl(threads, 256));
    if (a.vec)
      hipLaunchKernelGGL((mm_reduce_kernel<T, OT, ACT, 16 / sizeof(T)>), grid, dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL((mm_reduce_kernel<T, OT, ACT, 1>), grid, dim3(256), 0, st, a);
    EKYA_HIP(hipGetLastError());
  }
  return hipSuccess;
}

// Rows of a matrix copied to whole units, the rest of the last one zero.
template <typename T>
__global__ __launch_bounds__(256) void mm_pack_kernel(const T* p, long long ld, long long rows, int cols,
                                                      uint4* out) {
  constexpr int E = Elt<T>::E;
  const int units = cdiv(cols, E);
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, r = i / units;
  if (r >= rows) return;
  const int u = (int)(i - r * units);
  out[i] = load_any(p + r * ld + u * E, min(E, cols - u * E));
}

// An operand: `rows` rows of `cols` elements, ld apart.
struct MmMat {
  const void* p;
  long long ld, rows;
  int cols;
  bool units(int dt) const { return cols % dtype_vec(dt) == 0 && unit16(p, ld, dt); }
  int padded(int dt) const { return (int)cdivl(cols, dtype_vec(dt)) * dtype_vec(dt); }
  size_t pack_floats(int dt) const { return ((size_t)rows * padded(dt) * dtype_size(dt) + 15) / 16 * 4; }
};
template <typename T> hipError_t mm_copy(MmMat& m, float* ws, hipStream_t st) {
  const int dt = sizeof(T) == 2 ? DT_BF16 : DT_F32;
  const long long units = m.padded(dt) / Elt<T>::E, most = std::max(1LL, (1LL << 30) / units);
  for (long long r = 0; r < m.rows; r += most) {
    const long long n = std::min(most, m.rows - r);
    hipLaunchKernelGGL(mm_pack_kernel<T>, dim3((unsigned)cdivl(n * units, 256)), dim3(256), 0, st,
                       (const T*)m.p + r * m.ld, m.ld, n, m.cols, (uint4*)ws + r * units);
    EKYA_HIP(hipGetLastError());
  }
  m.p = ws;
  m.ld = m.cols = m.padded(dt);
  return hipSuccess;
}

// D from operands A and B (AOC, BOC: with the reduction as rows); a: all but
// the operands.
template <typename T, typename OT, bool AOC, bool BOC, int ACT>
hipError_t mm_product(MmArgs<T> a, const MmMat& A, const MmMat& B, hipStream_t st) {
  const int dt = sizeof(T) == 2 ? DT_BF16 : DT_F32;
  a.a = (const T*)A.p;
  a.lda = A.ld;
  a.b = (const T*)B.p;
  a.ldb = B.ld;
  a.Ra = A.cols;
  a.Cb = B.cols;
  return mm_run<T, OT, AOC, BOC, ACT>(a, A.units(dt) && B.units(dt), st);
}

size_t mm_forward_floats(const MatmulFwd& f) {
  const MmMat x{f.x, f.ldx, f.M, f.K}, w{f.w, f.ldw, f.N, f.K};
  const bool copy = mm_pack(f.dt == DT_F32, f.N, f.M, f.K);
  size_t n = mm_part_floats(f.N, f.M, f.K, f.dt, copy || (x.units(f.dt) && w.units(f.dt)));
  if (copy)
    n += (x.units(f.dt) ? 0 : x.pack_floats(f.dt)) + (w.units(f.dt) ? 0 : w.pack_floats(f.dt));
  return n;
}

template <typename T> hipError_t mm_forward(const MatmulFwd& f, float* ws, hipStream_t st) {
  const int dt = sizeof(T) == 2 ? DT_BF16 : DT_F32;
  MmMat x{f.x, f.ldx, f.M, f.K}, w{f.w, f.ldw, f.N, f.K};
  if (mm_pack(dt == DT_F32, f.N, f.M, f.K))
    for (MmMat* m : {&x, &w})
      if (!m->units(dt)) {
        const size_t n = m->pack_floats(dt);
        EKYA_HIP(mm_copy<T>(*m, ws, st));
        ws += n;
      }
  MmArgs<T> a{};
  a.R = f.N;
  a.C = f.M;
  a.Tn = f.K;
  a.bias = f.bias;
  a.res = (const T*)f.res;
  a.ldr = f.ldr;
  a.res_first = f.res && f.res_first;
  a.y = f.y;
  a.ldy = f.ldy;
  a.z = (T*)f.z;
  a.ldz = f.ldz;
  a.part = ws;
  a.vec = unit16(f.y, f.ldy, dt) && (!f.z || unit16(f.z, f.ldz, dt)) &&
          (!f.res || unit16(f.res, f.ldr, dt)) && reinterpret_cast<uintptr_t>(f.bias) % 16 == 0;
  return act_dispatch(f.act, [&](auto k) { return mm_product<T, T, false, false, k.value>(a, w, x, st); });
}

// ----------------------------------------------------------------- backward
// dz = dy act'(z), and the column sums of what is stored before its rounding.
// dz is rounded to T because both products take it as an operand of the matrix
// cores, whose rate in bf16 is 16 times that of fp32.
// A block takes a range of rows and up to 64 units of columns.
constexpr int DZ_NT = 256;
struct DzArgs {
  const void *dy, *z;
  void* dz;  // null: sums only
  long long lddy, ldz, lddz, M;
  int N, cu, cup, cchunks;
  long long rows;  // of a block
  float* part;     // [chunk][N] or null
};
template <typename T, int E, int ACT> __global__ __launch_bounds__(DZ_NT) void dz_kernel(DzArgs a) {
  __shared__ float red[DZ_NT * E];
  const int cc = blockIdx.x % a.cchunks;
  const long long chunk = blockIdx.x / a.cchunks;
  const int u = threadIdx.x & (a.cup - 1), rr = threadIdx.x / a.cup, rpp = DZ_NT / a.cup;
  const int c = (cc * a.cu + u) * E;
  const bool on = u < a.cu && c < a.N;
  const long long r1 = min(a.M, (chunk + 1) * a.rows);
  float s[E];
#pragma unroll
  for (int e = 0; e < E; ++e) s[e] = 0.f;
  if (on)
    for (long long r = chunk * a.rows + rr; r < r1; r += rpp) {
      float g[E], z[E];
      if constexpr (E > 1) {
        load_run((const T*)a.dy + r * a.lddy + c, g);
        if constexpr (ACT != ACT_NONE) load_run((const T*)a.z + r * a.ldz + c, z);
      } else {
        g[0] = to_f(((const T*)a.dy)[r * a.lddy + c]);
        if constexpr (ACT != ACT_NONE) z[0] = to_f(((const T*)a.z)[r * a.ldz + c]);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (ACT != ACT_NONE) g[e] = act_bwd<ACT, T>(g[e], z[e]);
        s[e] += g[e];
      }
      if (a.dz) {
        if constexpr (E > 1)
          store_run((T*)a.dz + r * a.lddz + c, g);
        else
          ((T*)a.dz)[r * a.lddz + c] = from_f<T>(g[0]);
      }
    }
  if (!a.part) return;
#pragma unroll
  for (int e = 0; e < E; ++e) red[threadIdx.x * E + e] = s[e];
  __syncthreads();
  for (int h = DZ_NT / 2; h >= a.cup; h >>= 1) {
    if ((int)threadIdx.x < h)
#pragma unroll
      for (int e = 0; e < E; ++e) red[threadIdx.x * E + e] += red[(threadIdx.x + h) * E + e];
    __syncthreads();
  }
  if (rr == 0 && on)
#pragma unroll
    for (int e = 0; e < E; ++e) a.part[chunk * a.N + c + e] = red[threadIdx.x * E + e];
}

// db[c] = sum over chunks: 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void db_kernel(const float* part, long long chunks, int N, float* db) {
  __shared__ float red[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  float s = 0.f;
  if (c < N)
#pragma unroll 8
    for (long long k = y; k < chunks; k += 32) s += part[k * N + c];
  red[y][x] = s;
  __syncthreads();
  for (int h = 16; h > 0; h >>= 1) {
    if (y < h) red[y][x] += red[y + h][x];
    __syncthreads();
  }
  if (y == 0 && c < N) db[c] = red[0][x];
}

// Rows of a block: 8 a thread at least, no more than 1024 blocks' worth of
// partial sums.
void dz_cut(DzArgs& a, int E) {
  const int units = cdiv(a.N, E);
  a.cchunks = cdiv(units, 64);
  a.cu = cdiv(units, a.cchunks);
  a.cup = 1;
  while (a.cup < a.cu) a.cup *= 2;
  const long long least = 8LL * (DZ_NT / a.cup);
  const long long want = std::max(1LL, 2048LL / a.cchunks);
  a.rows = std::max(least, cdivl(cdivl(a.M, std::min(1024LL, want)), least) * least);
}
size_t db_part_floats(long long M, int N, int E) {
  DzArgs a{};
  a.M = M;
  a.N = N;
  dz_cut(a, E);
  return (size_t)cdivl(M, a.rows) * N;
}

template <typename T, int E> hipError_t dz_run(DzArgs a, int act, float* db, hipStream_t st) {
  dz_cut(a, E);
  const long long chunks = cdivl(a.M, a.rows);
  if (chunks == 1 && db) {
    a.part = db;
    db = nullptr;
  }
  if (chunks) {
    EKYA_HIP(act_dispatch(act, [&](auto k) {
      hipLaunchKernelGGL((dz_kernel<T, E, k.value>), dim3((unsigned)(chunks * a.cchunks)), dim3(DZ_NT),
                         0, st, a);
      return hipGetLastError();
    }));
  }
  if (db) {
    hipLaunchKernelGGL(db_kernel, dim3(cdiv(a.N, 32)), dim3(1024), 0, st, a.part, chunks, a.N, db);
    EKYA_HIP(hipGetLastError());
  }
  return hipSuccess;
}

template <typename T> hipError_t mm_backward(const MatmulBwd& f, float* ws, hipStream_t st) {
  const int dt = sizeof(T) == 2 ? DT_BF16 : DT_F32;
  const bool act = f.act != ACT_NONE;
  const void* dz = act ? f.dz : f.dy;
  const long long lddz = act ? f.lddz : f.lddy;
  if (act || f.db) {
    DzArgs a{};
    a.dy = f.dy;
    a.lddy = f.lddy;
    a.z = f.z;
    a.ldz = f.ldz;
    a.dz = act ? f.dz : nullptr;
    a.lddz = f.lddz;
    a.M = f.M;
    a.N = f.N;
    a.part = f.db ? ws : nullptr;
    const bool unit = f.N % Elt<T>::E == 0 && unit16(f.dy, f.lddy, dt) &&
                      (!act || (unit16(f.z, f.ldz, dt) && unit16(f.dz, f.lddz, dt)));
    EKYA_HIP(unit ? (dz_run<T, Elt<T>::E>(a, f.act, f.db, st)) : (dz_run<T, 1>(a, f.act, f.db, st)));
  }
  MmMat g{dz, lddz, f.M, f.N};  // copied once for both products
  const bool copy_dx = f.dx && mm_pack(dt == DT_F32, f.K, f.M, f.N), copy_dw = f.dw && mm_pack(dt == DT_F32, f.K, f.N, f.M);
  MmMat packed = g;
  if ((copy_dx || copy_dw) && f.M > 0 && !g.units(dt)) {
    const size_t n = g.pack_floats(dt);
    EKYA_HIP(mm_copy<T>(packed, ws, st));
    ws += n;
  }
  auto other = [&](MmMat m, bool copy, float** rest, hipError_t* e) {
    *rest = ws;
    if (copy && !m.units(dt)) {
      const size_t n = m.pack_floats(dt);
      *e = mm_copy<T>(m, ws, st);
      *rest = ws + n;
    }
    return m;
  };
  hipError_t e = hipSuccess;
  if (f.dx && f.M > 0) {
    MmArgs<T> a{};
    const MmMat w = other({f.w, f.ldw, f.N, f.K}, copy_dx, &a.part, &e);
    EKYA_HIP(e);
    a.R = f.K;
    a.C = f.M;
    a.Tn = f.N;
    a.y = f.dx;
    a.ldy = f.lddx;
    a.vec = unit16(f.dx, f.lddx, dt);
    EKYA_HIP((mm_product<T, T, true, false, ACT_NONE>(a, w, copy_dx ? packed : g, st)));
  }
  if (f.dw) {
    MmArgs<T> a{};
    const MmMat x = other({f.x, f.ldx, f.M, f.K}, copy_dw && f.M > 0, &a.part, &e);
    EKYA_HIP(e);
    a.R = f.K;
    a.C = f.N;
    a.Tn = f.M;
    a.y = f.dw;
    a.ldy = f.K;
    const bool low = dt == DT_BF16 && f.dw_dt == DT_BF16;
    a.vec = unit16(f.dw, f.K, low ? DT_BF16 : DT_F32);
    const MmMat& b = copy_dw && f.M > 0 ? packed : g;
    EKYA_HIP(low ? (mm_product<T, T, true, true, ACT_NONE>(a, x, b, st))
                 : (mm_product<T, float, true, true, ACT_NONE>(a, x, b, st)));
  }
  return hipSuccess;
}

size_t mm_backward_floats(const MatmulBwd& f) {
  const bool act = f.act != ACT_NONE;
  const MmMat g{act ? f.dz : f.dy, act ? f.lddz : f.lddy, f.M, f.N}, x{f.x, f.ldx, f.M, f.K},
      w{f.w, f.ldw, f.N, f.K};
  const int dt = f.dt, E = dtype_vec(dt);
  const bool copy_dx = f.dx && mm_pack(dt == DT_F32, f.K, f.M, f.N), copy_dw = f.dw && mm_pack(dt == DT_F32, f.K, f.N, f.M);
  size_t n = 0, db = 0;
  if (f.dx)
    n = mm_part_floats(f.K, f.M, f.N, dt, copy_dx || (w.units(dt) && g.units(dt))) + (copy_dx && !w.units(dt) ? w.pack_floats(dt) : 0);
  if (f.dw)
    n = std::max(n, mm_part_floats(f.K, f.N, f.M, dt, copy_dw || (x.units(dt) && g.units(dt))) + (copy_dw && !x.units(dt) ? x.pack_floats(dt) : 0));
  if ((copy_dx || copy_dw) && !g.units(dt)) n += g.pack_floats(dt);
  // the bias gradient's partial sums are done with before the products begin
  if (f.db) db = std::max(db_part_floats(f.M, f.N, 1), f.N % E == 0 ? db_part_floats(f.M, f.N, E) : 0);
  return std::max(n, db);
}

}  // namespace

size_t matmul_workspace_floats(const MatmulFwd& f) { return mm_forward_floats(f); }
size_t matmul_backward_workspace_floats(const MatmulBwd& f) { return mm_backward_floats(f); }

hipError_t matmul_fwd(const MatmulFwd& f, float* ws, hipStream_t st) {
  return f.dt == DT_BF16 ? mm_forward<bf16>(f, ws, st) : mm_forward<float>(f, ws, st);
}

hipError_t matmul_bwd(const MatmulBwd& f, float* ws, hipStream_t st) {
  return f.dt == DT_BF16 ? mm_backward<bf16>(f, ws, st) : mm_backward<float>(f, ws, st);
}

}  // namespace ekya
