// The output layer with low-rank adapters: out[n] = W x[n] + b + s_g B_g (A_g x[n]).
//
// First u[n] = s_g A_g x[n] (32-bit sums), written as 16-bit terms whose sum
// has the mantissa the output needs, so that B_g u runs on the matrix
// instructions too: u = u_0 + u_1 (+ u_2), each the rounding of what the ones
// before left.  bfloat16 takes three terms (24 bits) for a 32-bit output and two
// for its own; half precision takes two (22 bits), where they do not hold a row as it
// is (terms_hold) of u divided by a power of two per row.
//
// Then W x in tiles of matrix instructions.  B_g u of a tile's one or two adapters are
// further steps of its product; of more it is added behind the product, as the bias
// is, and the rounding to the output's type comes as a tile is stored.  W is the
// matrix instruction's first operand and x its second, so that a lane holds
// consecutive outputs of one row.
#include <algorithm>

#include "wd_host.h"
#include "wd_num.h"
#include "wd_rows.h"

namespace wd {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef f32x4 __attribute__((aligned(2))) f32x4_any;

__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c, Bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c, Half) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

struct HeadArgs {
  wd_head h;
  const void* x;
  int64_t x_ld, N;
  const int32_t* adapter;  // NULL: none (also without adapters)
  void* out;
  int64_t out_ld;
  // [N][ul] terms of u, the rank padded to rp: term t of rank r at t * rp + r, uk of
  // them, zeros up to ul (a multiple of kStepK); zeros throughout for a row without an adapter
  uint16_t* u;
  float* us;               // [N] power of two that u was divided by
  int32_t rp, uk, ul;
  bool b16;                // B's rows start at multiples of 16 bytes
  bool stream;             // outputs past the caches
};

// Terms of u for an output of type O.
template <class T, class O>
constexpr int kTerms = 2;
template <>
constexpr int kTerms<Bf16, F32> = 3;

__device__ __forceinline__ int adapter_of(const HeadArgs& a, int64_t n) {
  if (!a.adapter || n >= a.N) return -1;
  const int g = a.adapter[n];
  return g >= 0 && g < a.h.n_adapters ? g : -1;
}

// Rows that do not end at a multiple of eight elements are read with loads that
// stay in the array: raw8 reads eight elements from p, or the array's last eight
// (at `last`) where that would pass its end, and fix8 moves them to their places and
// puts zeros from element n on.  Reads first, then the moves: several reads are under
// way together.  (Element by element, under a branch each, 78 rows of 1133 -> 1516 with
// as many adapters of rank 38 took 72 us for 60, 2548 of 67 -> 7042 41 for 36.)
// Arrays of fewer than eight elements (shorter_than_a_load) go to k_tiny.
template <class T>
__device__ __forceinline__ uint4 load8(const T* p) {
  return __builtin_bit_cast(uint4, *(const Few<T, 8>*)p);
}

template <class T>
__device__ __forceinline__ uint4 raw8(const T* p, const T* last) {
  return load8(p < last ? p : last);
}

template <class T>
__device__ __forceinline__ uint4 fix8(uint4 v, const T* p, int n, const T* last) {
  const int by = p > last ? (int)min(p - last, (ptrdiff_t)8) : 0;  // elements to move down
  uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
  if (by & 4) lo = hi, hi = 0;
  const int r = (by & 3) * 16;
  lo = lo >> r | (hi << 1) << (63 - r);
  hi >>= r;
  const auto low = [](int k) { return k >= 4 ? ~0ull : k <= 0 ? 0ull : (1ull << (16 * k)) - 1; };
  const int keep = by == 8 ? 0 : n;
  lo &= low(keep);
  hi &= low(keep - 4);
  return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

// The first n of eight elements, one by one, and zeros: for the largest tiles, which
// have no registers left to move elements in (64000 rows of 32 per adapter took 1470
// us with raw8 and fix8, and take 1220).
template <class T>
__device__ __forceinline__ uint4 few8(const T* p, int n) {
  if (n >= 8) return load8(p);
  Few<T, 8> v{};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) v.v[i] = p[i];
  return __builtin_bit_cast(uint4, v);
}

// The last eight elements of x, W, A and B.
template <class T>
__device__ __forceinline__ const T* last_x(const HeadArgs& a) {
  return (const T*)a.x + (a.N - 1) * a.x_ld + a.h.D - 8;
}
template <class T>
__device__ __forceinline__ const T* last_w(const HeadArgs& a) {
  return (const T*)a.h.weight + (a.h.P - 1) * a.h.weight_ld + a.h.D - 8;
}
template <class T>
__device__ __forceinline__ const T* last_a(const HeadArgs& a) {
  return (const T*)a.h.a + (int64_t)a.h.n_adapters * a.h.rank * a.h.D - 8;
}
template <class T>
__device__ __forceinline__ const T* last_b(const HeadArgs& a) {
  return (const T*)a.h.b + (int64_t)a.h.n_adapters * a.h.P * a.h.rank - 8;
}

// The terms of one value; an infinity or NaN is its first term.
template <class T, int TERMS>
__device__ __forceinline__ void split(float u, T* t) {
#pragma unroll
  for (int k = 0; k < TERMS; ++k) {
    t[k] = T::of(u);
    const float r = u - t[k].f();
    u = fabsf(r) < INFINITY ? r : 0.0f;  // (also where u is not finite)
  }
}

template <class T, int TERMS>
__device__ __forceinline__ void store_u(const HeadArgs& a, int64_t n, int r, float u) {
  T t[TERMS];
  split<T, TERMS>(u, t);
#pragma unroll
  for (int k = 0; k < TERMS; ++k) a.u[n * a.ul + k * a.rp + r] = t[k].u;
}

// Whether half precision's two terms hold u as it is: to 2^-16 of itself or 2^-22 of
// `parts`, the magnitudes of what its sum adds up (which 32-bit sums are off by as much
// for).  Their first is good to 11 bits and so is the second, but for its
// least place of 2^-24: a rank whose A x is small beside the row's others needs more.
template <class T>
__device__ __forceinline__ bool terms_hold(float u, float parts) {
  if constexpr (__is_same(T, Bf16)) {
    return true;
  } else {
    const float r = u - T::of(u).f(), e = r - T::of(r).f();
    return !(fabsf(e) > fmaxf(0x1p-16f * fabsf(u), 0x1p-22f * parts));  // (one that is not finite is its first term)
  }
}

// The power of two that a row's u are divided by: 1 for bfloat16, which has the
// range of 32 bits, and where half precision's two terms `hold` every u of the row.  Else
// one that puts the largest in [2^14, 2^15), so that what the terms leave of any is at
// most 2^-39 of the largest.
template <class T>
__device__ __forceinline__ float row_power(float largest, bool hold) {
  if constexpr (__is_same(T, Bf16)) {
    return 1.0f;
  } else {
    const uint32_t e = __float_as_uint(largest) & 0x7f800000u;
    if (e == 0 || (hold && largest < 0x1p15f)) return 1.0f;
    return fmaxf(__uint_as_float(e) * 0x1p-14f, 0x1p-70f);
  }
}

__device__ __forceinline__ float finite_abs(float u) { return fabsf(u) < INFINITY ? fabsf(u) : 0.0f; }

// The products of a row of n elements with two others, by a wavefront: each sum in two
// parts, in the lanes of even and of odd number.
template <class T>
__device__ __forceinline__ void row_products(const T* x, const T* sx, const T* w0, const T* w1, const T* sw, int n,
                                             float& s0, float& s1) {
  s0 = s1 = 0.0f;
#pragma unroll 2
  for (int k = (threadIdx.x & 63) * 8; k < n; k += 512) {
    uint4 xv, v0, v1;
    if (n % 8 == 0) {
      xv = load8(x + k), v0 = load8(w0 + k), v1 = load8(w1 + k);
    } else {
      xv = raw8(x + k, sx), v0 = raw8(w0 + k, sw), v1 = raw8(w1 + k, sw);
      xv = fix8(xv, x + k, n - k, sx);
      v0 = fix8(v0, w0 + k, n - k, sw);
      v1 = fix8(v1, w1 + k, n - k, sw);
    }
    const T *xe = (const T*)&xv, *e0 = (const T*)&v0, *e1 = (const T*)&v1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s0 = fmaf(xe[i].f(), e0[i].f(), s0);
      s1 = fmaf(xe[i].f(), e1[i].f(), s1);
    }
  }
  for (int o = 32; o > 1; o >>= 1) {
    s0 += __shfl_xor(s0, o);
    s1 += __shfl_xor(s1, o);
  }
}

// u[n]: a workgroup per row, a wavefront per rank at a time (two, whose reads are
// in flight together).
template <class T, int TERMS>
__global__ void __launch_bounds__(512) k_low_row(HeadArgs a) {
  __shared__ float us[WD_MAX_RANK], parts[WD_MAX_RANK];
  const int64_t n = blockIdx.x;
  const int g = adapter_of(a, n), D = a.h.D, R = a.h.rank;
  if (g < 0) {
    for (int k = threadIdx.x; k < a.ul; k += 512) a.u[n * a.ul + k] = 0;
    if (threadIdx.x == 0) a.us[n] = 1.0f;
    return;
  }
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T* x = (const T*)a.x + n * a.x_ld;
  const T* w = (const T*)a.h.a + (int64_t)g * R * D;
  const float sc = a.h.scale ? a.h.scale[g] : 1.0f;
  for (int r = wave * 2; r < R; r += 16) {
    float s0, s1;
    row_products(x, last_x<T>(a), w + (int64_t)r * D, w + (int64_t)min(r + 1, R - 1) * D, last_a<T>(a), D, s0, s1);
    const float t0 = __shfl_xor(s0, 1), t1 = __shfl_xor(s1, 1);
    if (lane < 2 && r + lane < R) {
      us[r + lane] = (lane ? s1 + t1 : s0 + t0) * sc;
      parts[r + lane] = (lane ? fabsf(s1) + fabsf(t1) : fabsf(s0) + fabsf(t0)) * fabsf(sc);
    }
  }
  __syncthreads();
  float top = 0.0f;
  bool hold = true;
  for (int r = lane; r < R; r += 64) {
    top = fmaxf(top, finite_abs(us[r]));
    hold &= terms_hold<T>(us[r], parts[r]);
  }
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float p = row_power<T>(top, __all(hold));
  if (threadIdx.x == 0) a.us[n] = p;
  if ((int)threadIdx.x < a.rp) store_u<T, TERMS>(a, n, threadIdx.x, (int)threadIdx.x < R ? us[threadIdx.x] / p : 0.0f);
  if (a.uk + (int)threadIdx.x < a.ul) a.u[n * a.ul + a.uk + threadIdx.x] = 0;
}

// u of 16 rows per workgroup by matrix instructions, the columns split between
// the wavefronts: A_g's ranks are the first operand, the rows the second, so
// that lane l holds four ranks of row l % 16 per block of 16 ranks.  Lanes read
// 32 consecutive bytes of their row, 128 of a row between them (the order of
// the columns in a sum of products is free).  The adapters of the 16 rows are
// taken one after another, each row keeping its own.  Rows of many adapters
// (more than kLowMix among 16) go one by one on the vector ALU instead.  (1024 rows of
// 1024 columns to 3000 outputs at rank 16, whole call: runs of 8 rows 41 us by matrix
// instructions and 63 one by one, an adapter per row 79 and 80.  In between the
// bound is low: runs of 4 rows would take 59 for 80, of 2 rows 60 for 74.)
constexpr int kLowMix = 3;

template <class T, int TERMS, int RB>
__global__ void __launch_bounds__(256) k_low_tile(HeadArgs a) {
  __shared__ float sums[4][16][RB * 16 + 1];  // [wavefront][row][rank]
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + col;
  const int D = a.h.D, R = a.h.rank;
  const int g = adapter_of(a, n);
  uint64_t todo = __ballot(g >= 0);
  int kinds = 0;
  for (uint64_t t = todo; t; ++kinds) t &= ~__ballot(g == __builtin_amdgcn_readlane(g, __ffsll((unsigned long long)t) - 1));
  if (kinds <= kLowMix) {
    const T* x = (const T*)a.x + (n < a.N ? n : a.N - 1) * a.x_ld;
    while (todo) {
      const int gg = __builtin_amdgcn_readlane(g, __ffsll((unsigned long long)todo) - 1);
      const bool mine = g == gg;
      todo &= ~__ballot(mine);
      f32x4 acc[RB] = {};
      const T* w[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) w[b] = (const T*)a.h.a + ((int64_t)gg * R + min(b * 16 + col, R - 1)) * D;
      // this wavefront's steps of 64 columns, the reads of some under way together
      constexpr int kSets = RB <= 2 ? 4 : RB <= 4 ? 2 : 1;
      const int k1 = wave * 64 + quad * 16, whole = (D - wave * 64) / 64 > 0 ? ((D - wave * 64) / 64 + 3) / 4 : 0;
      for (int i = 0; i < whole; i += kSets) {
        uint4 xv[kSets][2], wv[kSets][2][RB];
#pragma unroll
        for (int t = 0; t < kSets; ++t)
          if (i + t < whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int k = k1 + (i + t) * 256 + h * 8;
              xv[t][h] = load8(x + k);
#pragma unroll
              for (int b = 0; b < RB; ++b) wv[t][h][b] = load8(w[b] + k);
            }
          }
#pragma unroll
        for (int t = 0; t < kSets; ++t)
          if (i + t < whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int b = 0; b < RB; ++b) acc[b] = mfma16(wv[t][h][b], xv[t][h], acc[b], T{});
          }
      }
      const int k = k1 + whole * 256;
      if ((k & ~63) < D) {
        const T *sx = last_x<T>(a), *sa = last_a<T>(a);
        uint4 xv[2], wv[2][RB];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          xv[h] = raw8(x + k + h * 8, sx);
#pragma unroll
          for (int b = 0; b < RB; ++b) wv[h][b] = raw8(w[b] + k + h * 8, sa);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int left = D - k - h * 8;
          xv[h] = fix8(xv[h], x + k + h * 8, left, sx);
#pragma unroll
          for (int b = 0; b < RB; ++b) acc[b] = mfma16(fix8(wv[h][b], w[b] + k + h * 8, left, sa), xv[h], acc[b], T{});
        }
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (mine) sums[wave][col][b * 16 + quad * 4 + e] = acc[b][e];
    }
  } else {
    for (int i = wave; i < 16; i += 4) {
      const int gg = __builtin_amdgcn_readlane(g, i);
      if (gg < 0) continue;
      const T* x = (const T*)a.x + (n0 + i) * a.x_ld;
      const T* w = (const T*)a.h.a + (int64_t)gg * R * D;
      for (int r = 0; r < R; r += 2) {
        float s0, s1;
        row_products(x, last_x<T>(a), w + (int64_t)r * D, w + (int64_t)min(r + 1, R - 1) * D, last_a<T>(a), D, s0, s1);
        // (two parts, and zeros for the other two wavefronts')
        if (lane < 8 && r + (lane >> 2) < R) sums[lane & 3][i][r + (lane >> 2)] = lane & 2 ? 0.0f : lane & 4 ? s1 : s0;
      }
    }
  }
  __syncthreads();
  const int i = threadIdx.x >> 4, r0 = threadIdx.x & 15;
  const int gi = adapter_of(a, n0 + i);
  const float sc = gi >= 0 && a.h.scale ? a.h.scale[gi] : 1.0f;
  float u[RB], top = 0.0f;
  bool hold = true;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int r = b * 16 + r0;
    float q[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) q[w] = r < R ? sums[w][i][r] : 0.0f;
    u[b] = ((q[0] + q[1]) + (q[2] + q[3])) * sc;
    hold &= terms_hold<T>(u[b], (fabsf(q[0]) + fabsf(q[1]) + fabsf(q[2]) + fabsf(q[3])) * fabsf(sc));
    top = fmaxf(top, finite_abs(u[b]));
  }
  for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  hold = (__ballot(!hold) >> (lane & 48) & 0xffff) == 0;  // (of the row's 16 lanes)
  if (n0 + i >= a.N) return;
  const float p = gi < 0 ? 1.0f : row_power<T>(top, hold);
  if (r0 == 0) a.us[n0 + i] = p;
#pragma unroll
  for (int b = 0; b < RB; ++b)
    if (b * 16 + r0 < a.rp) store_u<T, TERMS>(a, n0 + i, b * 16 + r0, gi < 0 ? 0.0f : u[b] / p);
  for (int k = a.uk + r0; k < a.ul; k += 16) a.u[(n0 + i) * a.ul + k] = 0;
}

// A workgroup per row spreads few rows over the chip; from kLowRows on the rows
// share the reads of their adapter instead.  (1024 columns to 3000 outputs, rows in
// runs of 32, whole call: at rank 16 400 rows 17.0 us a workgroup each and 18.0 in
// tiles, 700 22.5 and 20.6, 2048 40 and 34; at rank 64 256 rows 22.3 and 24.2, 512 29.1
// and 29.3, 2048 76 and 58.  Rows of an adapter each stay faster by themselves: 2048 118
// and 141.)
constexpr int64_t kLowRows = 512;

template <class T, int TERMS>
void launch_low(const HeadArgs& a, hipStream_t s) {
  if (a.N < kLowRows) {
    hipLaunchKernelGGL((k_low_row<T, TERMS>), dim3((uint32_t)a.N), dim3(512), 0, s, a);
    return;
  }
  const dim3 grid((uint32_t)((a.N + 15) / 16)), block(256);
  if (a.h.rank <= 16)
    hipLaunchKernelGGL((k_low_tile<T, TERMS, 1>), grid, block, 0, s, a);
  else if (a.h.rank <= 32)
    hipLaunchKernelGGL((k_low_tile<T, TERMS, 2>), grid, block, 0, s, a);
  else if (a.h.rank <= 64)
    hipLaunchKernelGGL((k_low_tile<T, TERMS, 4>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_low_tile<T, TERMS, 8>), grid, block, 0, s, a);
}

// B_g u (before the row's power) of the four outputs from p on of one row per
// lane, on the vector ALU.
template <class T, int TERMS, int AHEAD>
__device__ __forceinline__ f32x4 low_of_row(const HeadArgs& a, int64_t n, int g, int p) {
  const int R = a.h.rank;
  f32x4 low = {0, 0, 0, 0};
  if (g < 0 || p >= a.h.P) return low;
  const T* b = (const T*)a.h.b + ((int64_t)g * a.h.P + p) * R;
  const uint16_t* ut = a.u + n * a.ul;
  const T* sb = last_b<T>(a);
  const int last = a.h.P - 1 - p;  // rows of B past the last are not read
  const auto add = [&](int r, const uint4 (&w)[4]) {
    uint4 t[TERMS];
#pragma unroll
    for (int k = 0; k < TERMS; ++k) t[k] = *(const uint4*)(ut + k * a.rp + r);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float u = ((const T*)&t[TERMS - 1])[i].f();
#pragma unroll
      for (int k = TERMS - 2; k >= 0; --k) u += ((const T*)&t[k])[i].f();
#pragma unroll
      for (int e = 0; e < 4; ++e) low[e] = fmaf(((const T*)&w[e])[i].f(), u, low[e]);
    }
  };
  uint4 w[4];
  int r = 0;
#pragma unroll AHEAD
  for (; r + 8 <= R; r += 8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = load8(b + (int64_t)min(e, last) * R + r);
    add(r, w);
  }
  if (r < R) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = raw8(b + (int64_t)min(e, last) * R + r, sb);
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = fix8(w[e], b + (int64_t)min(e, last) * R + r, R - r, sb);
    add(r, w);
  }
  return low;
}

// Whether one of the eight values is an infinity or NaN (all exponent bits set).
template <class T>
__device__ __forceinline__ bool not_finite(uint4 v) {
  constexpr uint32_t e = __is_same(T, Bf16) ? 0x7f80u : 0x7c00u;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad |= (w[i] & e) == e || (w[i] & (e << 16)) == (e << 16);
  return bad;
}

// A wavefront's rows of more adapters than this take the vector ALU, whose lanes
// each read their own row's B; the matrix instructions take the adapters in turn.
// (16384 rows of 1024 columns to 6000 outputs at rank 16, 128 rows a wavefront, whole
// call: 8 adapters among them 439 us in turn and 585 row by row, 16 653 and 612, 32 1092
// and 670.)
constexpr int kWaveMix = 16;

// B_g u for the wavefront's rows n0.., added to acc; prow(j, i) is the output of
// row i of operand block j, `ids` the rows' adapters, `mine` LDS of the
// wavefront's own, of 16 lane vectors or as many as it has accumulators.  A row's terms are zero for the other
// rows' adapters, so that a product with them adds nothing; where an adapter's
// weights are not all finite (and zero times them would be a NaN), its rows
// take the vector ALU.
template <class T, int TERMS, int TM, int TN, class PRow>
__device__ __forceinline__ void add_low(const HeadArgs& a, int64_t n0, const int* ids, PRow prow, f32x4* mine,
                                        f32x4 (&acc)[TM][TN]) {
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int R = a.h.rank, P = a.h.P;
  const int chunks = a.uk / 8, per = a.rp / 8;
  int g[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) g[i] = ids[i * 16 + col];
  uint64_t todo[TM];
  const auto start = [&]() {
#pragma unroll
    for (int i = 0; i < TM; ++i) todo[i] = __ballot(g[i] >= 0);
  };
  const auto next = [&]() {  // the first adapter left
    int gg = -1;
#pragma unroll
    for (int i = TM - 1; i >= 0; --i)
      if (todo[i]) gg = __builtin_amdgcn_readlane(g[i], __ffsll((unsigned long long)todo[i]) - 1);
#pragma unroll
    for (int i = 0; i < TM; ++i) todo[i] &= ~__ballot(g[i] == gg);
    return gg;
  };
  start();
  int kinds = 0;
  while (kinds <= kWaveMix && next() >= 0) ++kinds;
  if (kinds == 0) return;
  const bool all_by_row = kinds > kWaveMix;

  float us[TM];
  if constexpr (!__is_same(T, Bf16)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      us[i] = g[i] >= 0 ? a.us[n0 + i * 16 + col] : 1.0f;
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] *= 1.0f / us[i];  // (a power of two)
    }
  }
  // this lane's rows (bit i: of block i) that are left for the vector ALU
  uint32_t by_row = 0;
  const auto leave = [&](int gg) {
#pragma unroll
    for (int i = 0; i < TM; ++i) by_row |= (all_by_row ? g[i] >= 0 : g[i] == gg) << i;
  };
  constexpr bool kSlim = TM * TN >= 32;
  const T* sb = last_b<T>(a);
  const auto b_part = [&](int gg, int p, int r) {
    const T* b = (const T*)a.h.b + ((int64_t)gg * P + p) * R + r;
    return kSlim ? few8(b, R - r) : fix8(raw8(b, sb), b, R - r, sb);
  };
  const auto usable = [&](int gg) {  // whether an adapter's weights for these outputs are finite
    bool bad = false;
#pragma unroll 1
    for (int r = quad * 8; r < R; r += 32)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        bad |= not_finite<T>(b_part(gg, min(prow(j, col), P - 1), r));
    if (!__any(bad)) return true;
    leave(gg);
    return false;
  };
  start();
  int gg = -1;
  if (all_by_row)
    leave(-1);
  else
    do gg = next();
    while (gg >= 0 && per > 4 && !usable(gg));
#pragma unroll 1
  for (int kk = 0; gg >= 0;) {
    const int c = kk + quad, r = c < chunks ? (c % per) * 8 : 0;
    const T* B = (const T*)a.h.b + (int64_t)gg * P * R + r;
    uint4 b[TN], u[TM];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const T* from = B + (int64_t)min(prow(j, col), P - 1) * R;
      b[j] = kSlim ? few8(from, R - r) : raw8(from, sb);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t n = n0 + i * 16 + col;
      u[i] = *(const uint4*)(a.u + (n < a.N ? n : a.N - 1) * a.ul + c * 8);
    }
    if (!kSlim && R % 8) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = fix8(b[j], B + (int64_t)min(prow(j, col), P - 1) * R, R - r, sb);
    }
    if (per <= 4 && kk == 0) {  // (all of the adapter's columns are here)
      bool bad = false;
#pragma unroll
      for (int j = 0; j < TN; ++j) bad |= not_finite<T>(b[j]);
      if (__any(bad)) {
        leave(gg);
        kk = chunks;
      }
    }
    const bool used = kk + quad < chunks;
#pragma unroll
    for (int j = 0; j < TN; ++j)
      if (!used) b[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < TM; ++i)
      if (!used || g[i] != gg) u[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma16(b[j], u[i], acc[i][j], T{});
    kk += 4;
    if (kk >= chunks) {
      kk = 0;
      do gg = next();
      while (gg >= 0 && per > 4 && !usable(gg));
    }
  }
  if (__any(by_row != 0)) {
    // through LDS, so that the accumulators' indices are constants and they stay in registers
    constexpr int kHalf = TM * TN < 16 ? TM * TN : 16;
#pragma unroll
    for (int h = 0; h < TM * TN; h += kHalf) {
#pragma unroll 1
      for (int ij = h; ij < h + kHalf; ++ij) {
        const int64_t n = n0 + (ij / TN) * 16 + col;
        const int gi = by_row >> (ij / TN) & 1 ? ids[(ij / TN) * 16 + col] : -1;
        mine[(ij - h) * 64 + lane] = low_of_row<T, TERMS, 1>(a, n, gi, prow(ij % TN, quad * 4));
      }
#pragma unroll
      for (int ij = h; ij < h + kHalf; ++ij) acc[ij / TN][ij % TN] += mine[(ij - h) * 64 + lane];
    }
  }
  if constexpr (!__is_same(T, Bf16)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] *= us[i];
  }
}

// N consecutive outputs of a row, those from n on left out.
template <class O, int N>
__device__ __forceinline__ void store_out(O* out, const Few<O, N>& v, int n) {
  if (n >= N) {
    *(Few<O, N>*)out = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) out[i] = v.v[i];
  }
}

// The adapters' part and the bias, the rounding, and the store: a block of 16
// rows at a time through LDS (`mine`, the wavefront's own), so that a store
// instruction writes whole lines of a row.  In the accumulators' layout it writes
// 64 bytes (half as much of 16-bit outputs) of each of 16 rows: 64000 x 6000
// outputs of 32 bits took 1250 us, of 16 bits 962, and take 895 and 865.  Outputs
// larger than the caches go past them (`stream`: 864 and 856 us).
template <class T, class O, int TM, int TN>
__device__ __forceinline__ void finish_tile(const HeadArgs& a, int64_t n0, int p0, f32x4* mine, const int* ids, f32x4 (&acc)[TM][TN]) {
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4, P = a.h.P;
  if (ids) add_low<T, kTerms<T, O>>(a, n0, ids, [&](int j, int i) { return p0 + j * 16 + i; }, mine, acc);
  constexpr int kCols = TN * 16, kEach = 16 / sizeof(O);
  constexpr int kLine = kCols + kEach;  // a row in LDS, padded against bank conflicts
  constexpr int kLanes = kCols / kEach, kRows = 64 / kLanes;  // lanes of a row, rows of a store
  O* rows = (O*)mine;
  float bias[TN][4];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[j][e] = a.h.bias ? a.h.bias[min(p0 + j * 16 + quad * 4 + e, P - 1)] : 0.0f;
  const int c = (lane % kLanes) * kEach, r0 = lane / kLanes, left = P - p0 - c;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      Few<O, 4> v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v.v[e] = O::of(acc[i][j][e] + bias[j][e]);
      struct alignas(4 * sizeof(O)) Four {
        O v[4];
      };
      *(Four*)(rows + col * kLine + j * 16 + quad * 4) = __builtin_bit_cast(Four, v);
    }
#pragma unroll
    for (int q = 0; q < 16; q += kRows) {
      const uint4 v = *(const uint4*)(rows + (q + r0) * kLine + c);
      const int64_t n = n0 + i * 16 + q + r0;
      O* out = (O*)a.out + n * a.out_ld + p0 + c;
      if (n < a.N) {
        if (a.stream && left >= kEach)
          __builtin_nontemporal_store(__builtin_bit_cast(f32x4, v), (f32x4_any*)out);
        else
          store_out(out, __builtin_bit_cast(Few<O, kEach>, v), left);
      }
    }
  }
}

// 16 bytes per lane from `base` (the same in every lane) + the lane's offset
// straight to LDS at `to` + 16 * lane (the same `to` in every lane).  The compiler
// does not see this load (its builtin makes every LDS read wait for all of them):
// the data is there after loads_left() and a barrier.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to) {
  const uint64_t p = (uint64_t)base;  // (into scalar registers, where the compiler would not hold it there)
  base = (const void*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 |
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)p));
  // (m0 is a register that the compiler keeps to itself, and warns of here; it holds no
  // value there across other code, and is named so that none of its uses is put around this)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to)
               : "memory", "m0");
#pragma clang diagnostic pop
}
// Waits until at most N of this wavefront's loads are on their way (they arrive in order).
template <int N>
__device__ __forceinline__ void loads_left() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Few rows (16 * NB to a workgroup): what counts is that W streams through the chip once.
// A workgroup takes 32 outputs of every row, its eight wavefronts a part of the
// columns each; the operands come straight from memory (x from the caches), 128
// bytes of a row between the lanes, and the parts are added through LDS.
// With FEW rows (at most kFewRows) a workgroup first forms the rows' u itself,
// which costs it the reads of their adapters but the call a launch.
constexpr int kFewRows = 4;
template <class T, class O, int NB, bool FEW>
__global__ void __launch_bounds__(512) k_rows(HeadArgs a) {
  __shared__ f32x4 part[8][NB * 2][64];
  __shared__ float low_u[FEW ? kFewRows : 1][FEW ? WD_MAX_RANK : 1];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int D = a.h.D, P = a.h.P, p0 = blockIdx.x * 32, n0 = blockIdx.y * NB * 16;
  const T *w[2], *x[NB];
#pragma unroll
  for (int j = 0; j < 2; ++j) w[j] = (const T*)a.h.weight + (int64_t)min(p0 + j * 16 + col, P - 1) * a.h.weight_ld;
#pragma unroll
  for (int i = 0; i < NB; ++i) x[i] = (const T*)a.x + min<int64_t>(n0 + i * 16 + col, a.N - 1) * a.x_ld;
  // the row and the outputs that this lane finishes
  const int fi = n0 + (wave >> 1) * 16 + col, fp = p0 + (wave & 1) * 16 + quad * 4;
  const int g = wave < NB * 2 ? adapter_of(a, fi) : -1;
  struct Operands {
    uint4 w[2][2], x[2][NB];
  };
  const auto read = [&](int k, Operands& o) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 2; ++j) o.w[h][j] = load8(w[j] + k + h * 8);
#pragma unroll
      for (int i = 0; i < NB; ++i) o.x[h][i] = load8(x[i] + k + h * 8);
    }
  };
  f32x4 acc[NB][2] = {};
  const auto multiply = [&](const Operands& o) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mfma16(o.w[h][j], o.x[h][i], acc[i][j], T{});
  };
  // Two of this wavefront's steps of 64 columns are read at a time, the first two
  // before the adapter's part, so that they are under way together.
  const int step = 512, k1 = wave * 64 + quad * 16, whole = (D - wave * 64) / 64 > 0 ? ((D - wave * 64) / 64 + 7) / 8 : 0;
  Operands o0, o1;
  if (whole > 0) read(k1, o0);
  if (whole > 1) read(k1 + step, o1);
  f32x4 low = {0, 0, 0, 0};
  if constexpr (FEW) {
    const int R = a.h.rank, pairs = (R + 1) / 2;
    for (int i = wave; i < (int)a.N * pairs; i += 8) {
      const int n = i / pairs, r = i % pairs * 2, gn = adapter_of(a, n);
      if (gn < 0) continue;
      const T* w0 = (const T*)a.h.a + ((int64_t)gn * R + r) * D;
      float s0, s1;
      row_products((const T*)a.x + n * a.x_ld, last_x<T>(a), w0, w0 + (r + 1 < R ? D : 0), last_a<T>(a), D, s0, s1);
      const float sc = a.h.scale ? a.h.scale[gn] : 1.0f;
      const float t0 = __shfl_xor(s0, 1), t1 = __shfl_xor(s1, 1);
      if (lane < 2 && r + lane < R) low_u[n][r + lane] = (lane ? s1 + t1 : s0 + t0) * sc;
    }
    // (read behind the barrier below)
  } else if (g >= 0) {
    low = low_of_row<T, kTerms<T, O>, 2>(a, fi, g, fp);
    const float us = a.us[fi];
#pragma unroll
    for (int e = 0; e < 4; ++e) low[e] *= us;
  }
  if (whole > 0) multiply(o0);
  if (whole > 1) multiply(o1);
  for (int i = 2; i < whole; i += 2) {
    read(k1 + i * step, o0);
    if (i + 1 < whole) read(k1 + (i + 1) * step, o1);
    multiply(o0);
    if (i + 1 < whole) multiply(o1);
  }
  const int k = k1 + whole * step;
  if ((k & ~63) < D) {
    const T *sw = last_w<T>(a), *sx = last_x<T>(a);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < 2; ++j) o0.w[h][j] = raw8(w[j] + k + h * 8, sw);
#pragma unroll
      for (int i = 0; i < NB; ++i) o0.x[h][i] = raw8(x[i] + k + h * 8, sx);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int left = D - k - h * 8;
#pragma unroll
      for (int j = 0; j < 2; ++j) o0.w[h][j] = fix8(o0.w[h][j], w[j] + k + h * 8, left, sw);
#pragma unroll
      for (int i = 0; i < NB; ++i) o0.x[h][i] = fix8(o0.x[h][i], x[i] + k + h * 8, left, sx);
    }
    multiply(o0);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) part[wave][i * 2 + j][lane] = acc[i][j];
  __syncthreads();
  if (wave >= NB * 2) return;
  f32x4 y = part[0][wave][lane];
#pragma unroll
  for (int v = 1; v < 8; ++v) y += part[v][wave][lane];
  if (FEW && g >= 0 && fp < P) {
    const T* b = (const T*)a.h.b + ((int64_t)g * P + fp) * a.h.rank;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const T* be = b + (int64_t)min(e, P - 1 - fp) * a.h.rank;
      for (int r = 0; r < a.h.rank; r += 8) {
        const uint4 v = a.h.rank % 8 == 0 ? load8(be + r) : fix8(raw8(be + r, last_b<T>(a)), be + r, a.h.rank - r, last_b<T>(a));
#pragma unroll
        for (int i = 0; i < 8; ++i) low[e] = fmaf(((const T*)&v)[i].f(), r + i < a.h.rank ? low_u[fi][r + i] : 0.0f, low[e]);
      }
    }
  }
  y += low;
  if (fi >= a.N || fp >= P) return;
  Few<O, 4> out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out.v[e] = O::of(y[e] + (a.h.bias ? a.h.bias[min(fp + e, P - 1)] : 0.0f));
  store_out((O*)a.out + fi * a.out_ld + fp, out, P - fp);
}

constexpr int kStepK = 64;  // columns of a step: 128 bytes of a row

// Where chunk c (16 bytes) of tile row r lies in LDS: at c ^ swizzle, so that the
// 16 rows of an operand read fall on different banks.
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// The tile of this workgroup.  Workgroups go round the eight XCDs, each with an
// L2 of its own: an XCD takes a run of tiles, in groups of kGroup rows of tiles
// column by column, so that its workgroups share rows of x and of W.
constexpr uint32_t kGroup = 8;
__device__ __forceinline__ void my_tile(uint32_t rows, uint32_t cols, uint32_t& row, uint32_t& col) {
  const uint32_t all = rows * cols, xcd = blockIdx.x % 8, q = all / 8, r = all % 8;
  const uint32_t at = xcd * q + min(xcd, r) + blockIdx.x / 8;
  const uint32_t group = at / (kGroup * cols), first = group * kGroup, height = min(kGroup, rows - first);
  const uint32_t in = at - first * cols;
  col = in / height;
  row = first + in % height;
}

// Adapters of a tile that are steps of its product.  A step more costs a tile of 256
// rows 1.5 us, add_low about 2 per adapter with the first wait: 64 utterances of 1000 rows
// 938 us with one adapter in the steps, 906 with two; rows in runs of 32 lose with
// more (64000 rows: 1218 us by add_low, 1367 in up to eight steps).
constexpr int kKinds = 2;

// What a lane loads for the terms of another adapter's row.
__device__ const uint4 k_zeros[kStepK / 8] = {};

// BM rows and BN outputs per workgroup of WM x WN wavefronts.  Two steps of kStepK
// columns are in LDS.  A step is two halves: while one is multiplied, the next
// half's operands are read into registers; between the halves of a step every
// wavefront has read all of it, and the step after the next starts into its place.
template <class T, class O, int BM, int BN, int WM, int WN, bool ALIGNED>
__global__ void __launch_bounds__(64 * WM * WN, BM * BN / WM / WN > 8192 ? 1 : 2) k_project(HeadArgs a, uint32_t row_tiles, uint32_t col_tiles) {
  constexpr int kWaves_ = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr bool kSlim = BM * BN > 128 * 128;
  constexpr int kRowBytes = kStepK * 2, kChunks = kStepK / 8, kPartRows = 64 / kChunks;
  constexpr int kTile = (BM + BN) * kRowBytes;
  constexpr int kParts = kTile / 1024 / kWaves_;  // loads of a wavefront per step
  static_assert((BM / kPartRows) % kWaves_ == 0 && (BN / kPartRows) % kWaves_ == 0, "");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int D = a.h.D, P = a.h.P;
  uint32_t row_tile, col_tile;
  my_tile(row_tiles, col_tiles, row_tile, col_tile);
  const int64_t n0 = (int64_t)row_tile * BM;
  const int p0 = (int)col_tile * BN;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;

  // a step's loads of this wavefront: parts of BM rows of x, then of BN rows of W;
  // the lane's offset (bytes) in its row's part of the inputs
  const T* xt = (const T*)a.x + n0 * a.x_ld;
  const T* wt = (const T*)a.h.weight + (int64_t)p0 * a.h.weight_ld;
  uint32_t from[kParts];
  constexpr auto is_w = [](int i) { return i * kWaves_ * kPartRows >= BM; };
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const int row = (i * kWaves_ + wave) * kPartRows - (is_w(i) ? BM : 0) + lane / kChunks;
    const int64_t at = is_w(i) ? min(row, P - 1 - p0) * a.h.weight_ld : min<int64_t>(row, a.N - 1 - n0) * a.x_ld;
    from[i] = (uint32_t)((at + ((lane % kChunks) ^ swizzle(row)) * 8) * 2);
  }
  int* ids = (int*)(lds + 2 * kTile);  // the rows' adapters
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int full = ALIGNED ? D / kStepK * kStepK : 0;  // columns of whole steps, loaded straight to LDS
  const int main = (D + kStepK - 1) / kStepK * kStepK;
  // Rows that are not aligned for that go through registers, read a half step before
  // they are put in place.
  const auto source = [&](int k0, int i) {
    const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, k = k0 + ((lane % kChunks) ^ swizzle(row)) * 8;
    return k + (row < BM ? xt + min<int64_t>(row, a.N - 1 - n0) * a.x_ld : wt + (int64_t)min(row - BM, P - 1 - p0) * a.h.weight_ld);
  };
  uint4 held[ALIGNED ? 1 : kParts];
  int held_for = -1, held_k = 0;
  const auto stage_x = [&](int k0, int step) {
    if (k0 < full) {
#pragma unroll
      for (int i = 0; i < kParts; ++i)
        load_to_lds((is_w(i) ? wt : xt) + k0, from[i], __builtin_amdgcn_readfirstlane(lds0 + step + (i * kWaves_ + wave) * 1024));
    } else if constexpr (ALIGNED) {  // the last columns, zeros behind them
#pragma unroll 1
      for (int i = 0; i < kParts; ++i) {
        const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + step + (i * kWaves_ + wave) * 1024);
        const int64_t at = is_w(i) ? min(row - BM, P - 1 - p0) * a.h.weight_ld : min<int64_t>(row, a.N - 1 - n0) * a.x_ld;
        if (k0 + c * 8 < D)
          load_to_lds((is_w(i) ? wt : xt) + k0, (uint32_t)((at + c * 8) * 2), to);
        else
          load_to_lds(k_zeros, (uint32_t)c * 16, to);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kParts; ++i) held[i] = is_w(i) ? raw8(source(k0, i), last_w<T>(a)) : raw8(source(k0, i), last_x<T>(a));
      held_for = step;
      held_k = k0;
    }
  };
  const auto put = [&]() {  // what was fetched, to its place
    if constexpr (!ALIGNED) {
      if (held_for < 0) return;
      if (held_k + kStepK > D) {  // (the row's last columns)
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, k = held_k + ((lane % kChunks) ^ swizzle(row)) * 8;
          held[i] = is_w(i) ? fix8(held[i], source(held_k, i), D - k, last_w<T>(a)) : fix8(held[i], source(held_k, i), D - k, last_x<T>(a));
        }
      }
#pragma unroll
      for (int i = 0; i < kParts; ++i) *(uint4*)(lds + held_for + (i * kWaves_ + wave) * 1024 + lane * 16) = held[i];
      held_for = -1;
    }
  };
  stage_x(0, 0);
  put();

  // Rows of a few adapters: each adapter's B_g u is a step (or a few) more, of u's
  // terms and B's columns, whose loads are under way while W x is still multiplied;
  // the other adapters' rows have zeros for their terms there.
  int steps = main;
  bool one = false, mixed = false;  // all rows of one adapter; rows left for add_low
  if (a.adapter) {
    int g[BM / 64], kinds = 0, least = 0;
    bool fits = a.rp <= kStepK;
    uint64_t todo[BM / 64];
#pragma unroll
    for (int q = 0; q < BM / 64; ++q) {
      const int64_t n = n0 + q * 64 + lane;
      g[q] = adapter_of(a, n);
      if (wave == 0) ids[q * 64 + lane] = g[q];
      if (!__is_same(T, Bf16) && g[q] >= 0) fits &= a.us[n] == 1.0f;
      if (g[q] < 0 && n < a.N) least = -1;
      todo[q] = __ballot(g[q] >= 0);
    }
    for (; kinds <= kKinds; ++kinds) {
      int gg = -1;
#pragma unroll
      for (int q = 0; q < BM / 64; ++q)
        if (todo[q]) gg = __builtin_amdgcn_readlane(g[q], __ffsll((unsigned long long)todo[q]) - 1);
      if (gg < 0) break;
#pragma unroll
      for (int q = 0; q < BM / 64; ++q) todo[q] &= ~__ballot(g[q] == gg);
      if (threadIdx.x == 0 && kinds < kKinds) ids[BM + kinds] = gg;
    }
    if (kinds > 0) {
      one = kinds == 1 && __all(least == 0);
      mixed = kinds > kKinds || !__all(fits);
      if (!mixed) {
        // zeros times an infinite weight would be a NaN: in another adapter's row, and in
        // the adapter's own, whose later terms may be zero
        __syncthreads();
        const int per = a.rp / 8;
        bool bad = false;
        for (int i = threadIdx.x; i < kinds * BN * per; i += 64 * kWaves_) {
          const int r = i % per * 8, p = min(p0 + i / per % BN, P - 1), gg = ids[BM + i / per / BN];
          const T* b = (const T*)a.h.b + ((int64_t)gg * P + p) * a.h.rank + r;
          bad |= not_finite<T>(kSlim ? few8(b, a.h.rank - r) : fix8(raw8(b, last_b<T>(a)), b, a.h.rank - r, last_b<T>(a)));
        }
        mixed = __syncthreads_or(bad);
      }
      if (!mixed) steps += a.ul * kinds;
    }
    __syncthreads();
  }
  const auto stage = [&](int k0, int step) {
    if (k0 < main) return stage_x(k0, step);
    const int gg = __builtin_amdgcn_readfirstlane(ids[BM + (k0 - main) / a.ul]), at = (k0 - main) % a.ul;
    const int c0 = at / 8, per = a.rp / 8, chunks = a.uk / 8, R = a.h.rank;
    const uint16_t* ut = a.u + n0 * a.ul + at;
    const T* bt = (const T*)a.h.b + ((int64_t)gg * P + p0) * R;
#pragma unroll 1
    for (int i = 0; i < kParts; ++i) {
      const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
      const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + step + (i * kWaves_ + wave) * 1024);
      if (is_w(i)) {
        const int r = c0 + c < chunks ? (c0 + c) % per * 8 : 0;  // (past the terms, u is zero)
        const T* b = bt + (int64_t)min(row - BM, P - 1 - p0) * R + r;
        if (a.b16)
          load_to_lds(bt, (uint32_t)((b - bt) * 2), to);
        else if (kSlim)
          *(uint4*)(lds + step + (i * kWaves_ + wave) * 1024 + lane * 16) = few8(b, R - r);
      } else if (one || ids[row] == gg) {
        load_to_lds(ut, (uint32_t)((min<int64_t>(row, a.N - 1 - n0) * a.ul + c * 8) * 2), to);
      } else {
        load_to_lds(k_zeros, (uint32_t)c * 16, to);
      }
    }
    if (!kSlim && !a.b16) {  // (B's rows through registers, where there are some to spare their reads under way together)
      uint4 v[kParts];
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
        const int r = c0 + c < chunks ? (c0 + c) % per * 8 : 0;
        if (is_w(i)) v[i] = raw8(bt + (int64_t)min(row - BM, P - 1 - p0) * R + r, last_b<T>(a));
      }
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const int row = (i * kWaves_ + wave) * kPartRows + lane / kChunks, c = (lane % kChunks) ^ swizzle(row);
        const int r = c0 + c < chunks ? (c0 + c) % per * 8 : 0;
        if (is_w(i))
          *(uint4*)(lds + step + (i * kWaves_ + wave) * 1024 + lane * 16) =
              fix8(v[i], bt + (int64_t)min(row - BM, P - 1 - p0) * R + r, R - r, last_b<T>(a));
      }
    }
  };

  f32x4 acc[TM][TN] = {};
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  struct Operands {
    uint4 w[TN], x[TM];
  } even, odd;
  const int read_at = (lane & 15) * kRowBytes + (((lane >> 4) ^ swizzle(lane & 15)) << 4);
  const auto read = [&](int step, int half, Operands& o) {
    const int at = step + (read_at ^ (half << 6));
#pragma unroll
    for (int j = 0; j < TN; ++j) o.w[j] = *(const uint4*)(lds + at + (BM + wn + j * 16) * kRowBytes);
#pragma unroll
    for (int i = 0; i < TM; ++i) o.x[i] = *(const uint4*)(lds + at + (wm + i * 16) * kRowBytes);
  };
  const auto multiply = [&](const Operands& o) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma16(o.w[j], o.x[i], acc[i][j], T{});
    // an operand read between every few products
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, TM * TN / (TM + TN), 0);
    }
  };
  int now = 0, next = kTile;
  if (kStepK < steps) {
    stage(kStepK, next);
    put();
    kStepK < full ? loads_left<kParts>() : loads_left<0>();
  } else {
    loads_left<0>();
  }
  __syncthreads();
  read(now, 0, even);
  // (One copy of the products and no branch around them: with more the compiler
  // holds the accumulators twice.  The last step's reads of a next one are of no use.)
  for (int k0 = 0; k0 < steps; k0 += kStepK) {
    read(now, 1, odd);
    multiply(even);
    put();
    loads_left<0>();
    __syncthreads();  // this step has been read, the next one is there
    if (k0 + 2 * kStepK < steps) stage(k0 + 2 * kStepK, now);
    read(next, 0, even);
    multiply(odd);
    now = next;
    next = kTile - next;
  }
  finish_tile<T, O>(a, n0 + wm, p0 + wn, (f32x4*)lds + wave * (TM * TN < 16 ? TM * TN : 16) * 64, mixed ? ids + wm : nullptr, acc);
}

template <class T, class O, int BM, int BN, int WM, int WN, bool ALIGNED>
void launch_tiles(const HeadArgs& a, hipStream_t s) {
  const uint32_t rows = (uint32_t)((a.N + BM - 1) / BM), cols = ((uint32_t)a.h.P + BN - 1) / BN;
  auto* k = k_project<T, O, BM, BN, WM, WN, ALIGNED>;
  constexpr int each = BM * BN / 256 / (WM * WN), low = (each < 16 ? each : 16) * 1024 * WM * WN;  // (add_low's)
  constexpr int stages = 2 * (BM + BN) * kStepK * 2;
  static_assert(low <= stages, "");
  constexpr int bytes = stages + (BM + kKinds) * 4;
  static std::atomic<uint64_t> done{0};
  allow_lds((const void*)k, bytes, done);
  hipLaunchKernelGGL(k, dim3(rows * cols), dim3(64 * WM * WN), bytes, s, a, rows, cols);
}

// A thread per output, for heads whose arrays are too small for loads of eight
// elements: the formula as it stands.
template <class T, class O>
__global__ void __launch_bounds__(256) k_tiny(HeadArgs a) {
  const int D = a.h.D, R = a.h.rank;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.N * a.h.P; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / a.h.P;
    const int p = (int)(i % a.h.P), g = adapter_of(a, n);
    const T *x = (const T*)a.x + n * a.x_ld, *w = (const T*)a.h.weight + p * a.h.weight_ld;
    float y = 0.0f, low = 0.0f;
    for (int k = 0; k < D; ++k) y = fmaf(x[k].f(), w[k].f(), y);
    for (int r = 0; g >= 0 && r < R; ++r) {
      const T* ar = (const T*)a.h.a + ((int64_t)g * R + r) * D;
      float u = 0.0f;
      for (int k = 0; k < D; ++k) u = fmaf(x[k].f(), ar[k].f(), u);
      low = fmaf(a.h.scale ? a.h.scale[g] * u : u, ((const T*)a.h.b)[((int64_t)g * a.h.P + p) * R + r].f(), low);
    }
    ((O*)a.out)[n * a.out_ld + p] = O::of(y + low + (a.h.bias ? a.h.bias[p] : 0.0f));
  }
}

template <class T, class O>
void launch_project(HeadArgs a, hipStream_t s) {
  const int64_t GR = a.adapter ? (int64_t)a.h.n_adapters * a.h.rank : kLoad;
  if (shorter_than_a_load(a.N, a.x_ld, a.h.D) || shorter_than_a_load(a.h.P, a.h.weight_ld, a.h.D) ||
      shorter_than_a_load(GR, a.h.D, a.h.D) || shorter_than_a_load(GR, a.h.P, a.h.P)) {
    const uint64_t blocks = ((uint64_t)a.N * a.h.P + 255) / 256;
    hipLaunchKernelGGL((k_tiny<T, O>), dim3((uint32_t)std::min<uint64_t>(blocks, 1 << 16)), dim3(256), 0, s, a);
    return;
  }
  const dim3 outs(((uint32_t)a.h.P + 31) / 32), block(512);
  if (a.adapter && a.N <= kFewRows) {
    hipLaunchKernelGGL((k_rows<T, O, 1, true>), outs, block, 0, s, a);
    return;
  }
  if (a.adapter) {
    constexpr int terms = kTerms<T, O>;
    a.uk = terms * a.rp;
    a.ul = (a.uk + kStepK - 1) / kStepK * kStepK;
    a.b16 = a.h.rank % 8 == 0 && !((uintptr_t)a.h.b & 15);
    launch_low<T, terms>(a, s);
  }
  // (the loads straight to LDS: 16 bytes, 32-bit offsets within a tile)
  const bool aligned = a.h.D % 8 == 0 && a.x_ld < (1 << 22) && a.h.weight_ld < (1 << 22) && a.x_ld % 8 == 0 && a.h.weight_ld % 8 == 0 && !((uintptr_t)a.x & 15) &&
                       !((uintptr_t)a.h.weight & 15);
  a.stream = (uint64_t)a.N * a.h.P * sizeof(O) >= (256u << 20);
  const auto tiles = [&](int64_t m, int64_t n) { return ((a.N + m - 1) / m) * ((a.h.P + n - 1) / n); };
  // Rows of many adapters each in a small output stay with k_rows while its workgroups
  // are one per compute unit at most: 128 rows of as many adapters, 512 -> 3000, take
  // 13.0 us and in tiles 18.8, 256 of 300 -> 1500 13.3 and 20.5; past that the tiles
  // are ahead (256 of 1024 -> 6000 33 us for 41), and for rows of one adapter throughout
  // (128 of 1133 -> 1516 24 us for 30).  Which adapters the rows use is known on the
  // device only: the rule counts those that the head holds, so that 128 rows of one
  // adapter take 24.0 us with a head of 20 adapters or 1000 and 20.5 with one of four.
  const bool many = a.adapter && (int64_t)a.h.n_adapters * 16 > a.N;
  const int64_t blocks64 = (a.N + 63) / 64;
  if (a.N <= 16)
    hipLaunchKernelGGL((k_rows<T, O, 1, false>), outs, block, 0, s, a);
  else if (a.N <= 32)
    hipLaunchKernelGGL((k_rows<T, O, 2, false>), outs, block, 0, s, a);
  else if (a.N <= 64 || (many && outs.x * blocks64 <= 256))
    hipLaunchKernelGGL((k_rows<T, O, 4, false>), dim3(outs.x, (uint32_t)blocks64), block, 0, s, a);
  else if (!aligned && tiles(128, 128) >= 192)
    launch_tiles<T, O, 128, 128, 2, 2, false>(a, s);
  else if (!aligned)
    launch_tiles<T, O, 64, 64, 2, 2, false>(a, s);
  else if (tiles(256, 256) >= 256)
    launch_tiles<T, O, 256, 256, 2, 4, true>(a, s);
  else if (tiles(128, 128) >= 192)
    launch_tiles<T, O, 128, 128, 2, 2, true>(a, s);
  else
    launch_tiles<T, O, 64, 64, 2, 2, true>(a, s);
}

}  // namespace wd

using namespace wd;

static wd_status check_head(const wd_head* h) {
  if (!h) return fail(WD_EINVAL, "project: null head");
  if (h->D < 1) return fail(WD_EINVAL, "project: D must be >= 1");
  if (h->P < 1 || h->P >= (1 << 24)) return fail(WD_EINVAL, "project: P out of range");
  if (h->type != WD_F16 && h->type != WD_BF16) return fail(WD_EINVAL, "project: type must be WD_F16 or WD_BF16");
  if (h->weight_ld < h->D) return fail(WD_EINVAL, "project: weight_ld below D");
  if (!h->weight) return fail(WD_EINVAL, "project: null weight");
  if (h->n_adapters < 0) return fail(WD_EINVAL, "project: negative n_adapters");
  if (h->n_adapters > 0) {
    if (h->rank < 1 || h->rank > WD_MAX_RANK) return fail(WD_EINVAL, "project: rank out of range");
    if (!h->a || !h->b) return fail(WD_EINVAL, "project: null adapter weights");
  }
  if ((uintptr_t)h->weight & 1 || (uintptr_t)h->a & 1 || (uintptr_t)h->b & 1 || (uintptr_t)h->bias & 3 ||
      (uintptr_t)h->scale & 3)
    return fail(WD_EINVAL, "project: misaligned weights");
  return WD_OK;
}

constexpr int64_t kMostRows = 1 << 27;  // rows of a launch

// Workspace: the terms of u (at most three), then the rows' powers of two.
static int padded_rank(const wd_head* h) { return (h->rank + 7) / 8 * 8; }
static size_t u_bytes(const wd_head* h, int64_t N) { return align_up((uint64_t)N * ((3 * padded_rank(h) + 63) / 64 * 64) * 2, 256); }
static size_t project_bytes(const wd_head* h, int64_t N) {
  N = std::min(N, kMostRows);
  return h->n_adapters > 0 ? u_bytes(h, N) + align_up((uint64_t)N * sizeof(float), 256) : 0;
}

extern "C" wd_status wd_project_workspace_bytes(const wd_head* h, int64_t N, size_t* bytes) {
  if (!bytes) return fail(WD_EINVAL, "project_workspace_bytes: null output");
  wd_status st = check_head(h);
  if (st != WD_OK) return st;
  if (N < 0 || N > INT32_MAX) return fail(WD_EINVAL, "project: N out of range");
  *bytes = project_bytes(h, N);
  return WD_OK;
}

extern "C" wd_status wd_project(const wd_head* h, const void* x, int64_t x_ld, int64_t N, const int32_t* adapter,
                                void* out, int64_t out_ld, int32_t out_type, void* ws, size_t ws_bytes, void* stream) {
  wd_status st = check_head(h);
  if (st != WD_OK) return st;
  if (N < 0 || N > INT32_MAX) return fail(WD_EINVAL, "project: N out of range");
  if (out_type != WD_F32 && out_type != h->type) return fail(WD_EINVAL, "project: out_type must be WD_F32 or the head's type");
  if (x_ld < h->D || out_ld < h->P) return fail(WD_EINVAL, "project: row stride too small");
  if (N == 0) return WD_OK;
  if (!x || !out) return fail(WD_EINVAL, "project: null rows or output");
  if ((uintptr_t)x & 1 || (uintptr_t)out & (out_type == WD_F32 ? 3 : 1) || (uintptr_t)adapter & 3)
    return fail(WD_EINVAL, "project: misaligned array");
  if (h->n_adapters == 0) adapter = nullptr;
  const size_t need = adapter ? project_bytes(h, N) : 0;
  if (need && (!ws || ws_bytes < need || (uintptr_t)ws & 255))
    return fail(WD_EINVAL, "project: workspace missing, too small or not 256-byte aligned");
  if (((uint64_t)N + 63) / 64 * (((uint64_t)h->P + 63) / 64) > INT32_MAX)
    return fail(WD_EINVAL, "project: too many rows for one call");
  hipStream_t s = (hipStream_t)stream;
  // (a launch has fewer than 2^32 threads: 2^28 rows in tiles of 16 are as many)
  for (int64_t n0 = 0; n0 < N; n0 += kMostRows) {
    const int64_t n = std::min(kMostRows, N - n0);
    HeadArgs a{*h, (const uint16_t*)x + n0 * x_ld, x_ld, n, adapter ? adapter + n0 : nullptr,
               (char*)out + n0 * out_ld * (out_type == WD_F32 ? 4 : 2), out_ld, (uint16_t*)ws,
               adapter ? (float*)((char*)ws + u_bytes(h, n)) : nullptr, adapter ? padded_rank(h) : 0, 0, 0, false, false};
    if (h->type == WD_F16)
      out_type == WD_F32 ? launch_project<Half, F32>(a, s) : launch_project<Half, Half>(a, s);
    else
      out_type == WD_F32 ? launch_project<Bf16, F32>(a, s) : launch_project<Bf16, Bf16>(a, s);
  }
  return hip_check(hipGetLastError(), "project");
}
