// The output layer with low-rank adapters: out[n] = W x[n] + b + s_g B_g (A_g x[n]).
//
// First u[n] = s_g A_g x[n] (32-bit sums), written as 16-bit terms whose sum
// has the mantissa the output needs, so that B_g u runs on the matrix
// instructions too: u = u_0 + u_1 (+ u_2), each the rounding of what the ones
// before left.  bfloat16 takes three terms (24 bits) for a 32-bit output and two
// for its own; half precision takes two (22 bits), of u divided by a power of two
// per row that puts the row's largest u in [1, 2).
//
// Then W x in tiles of matrix instructions; the adapters' part, the bias and the
// rounding to the output's type are added as a tile is stored.  W is the
// matrix instruction's first operand and x its second, so that a lane holds
// consecutive outputs of one row.
#include "wd_host.h"
#include "wd_num.h"

namespace wd {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

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
  uint16_t* u;             // [N][uk] terms of u, rank padded to rp: term t of rank r at t * rp + r
  float* us;               // [N] power of two that u was divided by (half precision)
  int32_t rp, uk;
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

// Eight elements at p, those from `n` on as zero.
template <class T>
__device__ __forceinline__ uint4 load8(const T* p, int n) {
  if (n >= 8) return __builtin_bit_cast(uint4, *(const Few<T, 8>*)p);
  Few<T, 8> v{};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) v.v[i] = p[i];
  return __builtin_bit_cast(uint4, v);
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

// u of 64 rows' worth of lanes: lane l holds the sums of rank r of its row in
// s[r / step] ... written by the callers below.
template <class T, int TERMS>
__device__ __forceinline__ void store_u(const HeadArgs& a, int64_t n, int r, float u) {
  T t[TERMS];
  split<T, TERMS>(u, t);
#pragma unroll
  for (int k = 0; k < TERMS; ++k) a.u[n * a.uk + k * a.rp + r] = t[k].u;
}

// The power of two that a row's u are divided by: 1 for bfloat16.
template <class T>
__device__ __forceinline__ float row_power(float largest) {
  if constexpr (sizeof(T) && __is_same(T, Bf16)) return 1.0f;
  const uint32_t e = __float_as_uint(largest) & 0x7f800000u;
  return e == 0 || e >= 0x7e800000u ? (e == 0 ? 1.0f : 0x1p126f) : __uint_as_float(e);
}

// u[n]: a workgroup per row, a wavefront per rank at a time.
template <class T, int TERMS>
__global__ void __launch_bounds__(256) k_low_row(HeadArgs a) {
  __shared__ float us[WD_MAX_RANK];
  const int64_t n = blockIdx.x;
  const int g = adapter_of(a, n), D = a.h.D, R = a.h.rank;
  if (g < 0) return;  // (never read)
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T* x = (const T*)a.x + n * a.x_ld;
  const float sc = a.h.scale ? a.h.scale[g] : 1.0f;
  for (int r = wave; r < R; r += 4) {
    const T* w = (const T*)a.h.a + ((int64_t)g * R + r) * D;
    float s = 0.0f;
    for (int k = lane * 8; k < D; k += 512) {
      const uint4 xv = load8(x + k, D - k), wv = load8(w + k, D - k);
      const T *xe = (const T*)&xv, *we = (const T*)&wv;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(xe[i].f(), we[i].f(), s);
    }
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) us[r] = s * sc;
  }
  __syncthreads();
  float top = 0.0f;
  for (int r = 0; r < R; ++r) top = fmaxf(top, fabsf(us[r]) < INFINITY ? fabsf(us[r]) : 0.0f);
  const float p = row_power<T>(top);
  if (threadIdx.x == 0) a.us[n] = p;
  for (int r = threadIdx.x; r < a.rp; r += 256) store_u<T, TERMS>(a, n, r, r < R ? us[r] / p : 0.0f);
}

// A lane's address for tile rows past the end of the inputs' columns.
__device__ uint4 k_zeros;

// The part of B_g u for the lane's rows, added to acc; `which(i)` is the row of
// block i that the lane holds, `prow(j)` the output whose weights it reads.
template <class T, int TM, int TN, class PRow>
__device__ __forceinline__ void add_low(const HeadArgs& a, int64_t n0, PRow prow, f32x4 (&acc)[TM][TN]) {
  const int lane = threadIdx.x & 63;
  const int R = a.h.rank, P = a.h.P;
  int g[TM];
  float us[TM];
  uint64_t any = 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t n = n0 + i * 16 + (lane & 15);
    g[i] = adapter_of(a, n);
    us[i] = g[i] >= 0 ? a.us[n] : 0.0f;
    any |= __ballot(g[i] >= 0);
  }
  if (!any) return;
  const int chunks = a.uk / 8, per = a.rp / 8;
  for (int kk = 0; kk < chunks; kk += 4) {
    const int c = kk + (lane >> 4), r = (c % per) * 8;
    uint4 u[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      u[i] = make_uint4(0, 0, 0, 0);
      if (g[i] >= 0 && c < chunks) u[i] = *(const uint4*)(a.u + (n0 + i * 16 + (lane & 15)) * a.uk + c * 8);
    }
    // the adapters of the rows, one after another
    uint64_t todo[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) todo[i] = __ballot(g[i] >= 0);
    for (;;) {
      int gg = -1;
#pragma unroll
      for (int i = TM - 1; i >= 0; --i)
        if (todo[i]) gg = __builtin_amdgcn_readlane(g[i], __ffsll((unsigned long long)todo[i]) - 1);
      if (gg < 0) break;
      uint4 b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int p = prow(j);
        b[j] = make_uint4(0, 0, 0, 0);
        if (c < chunks && p < P) b[j] = load8((const T*)a.h.b + ((int64_t)gg * P + p) * R + r, R - r);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const bool mine = g[i] == gg;
        const uint64_t m = __ballot(mine);
        todo[i] &= ~m;
        if (!m) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const f32x4 t = mfma16(b[j], u[i], f32x4{0, 0, 0, 0}, T{});
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = mine ? fmaf(t[e], us[i], acc[i][j][e]) : acc[i][j][e];
        }
      }
    }
  }
}

// Four (or, of 16-bit outputs, eight) consecutive outputs of a row.
template <class O, int N>
__device__ __forceinline__ void store_out(O* out, const float* y, int n) {
  Few<O, N> v;
#pragma unroll
  for (int i = 0; i < N; ++i) v.v[i] = O::of(y[i]);
  if (n >= N) {
    *(Few<O, N>*)out = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) out[i] = v.v[i];
  }
}

// Which of a wavefront's outputs the lane's row i (0..15) of operand block j
// is: chosen so that the blocks a lane holds are consecutive outputs, 16 bytes
// at a store.
template <class O>
__device__ __forceinline__ int out_of(int j, int i) {
  if constexpr (sizeof(O) == 4) return j * 16 + i;
  return (j >> 1) * 32 + (i >> 2) * 8 + (j & 1) * 4 + (i & 3);
}

template <class T, class O, int TM, int TN>
__device__ __forceinline__ void finish_tile(const HeadArgs& a, int64_t n0, int p0, f32x4 (&acc)[TM][TN]) {
  const int lane = threadIdx.x & 63, P = a.h.P;
  if (a.adapter) add_low<T>(a, n0, [&](int j) { return p0 + out_of<O>(j, lane & 15); }, acc);
  constexpr int W = sizeof(O) == 4 ? 1 : 2;  // blocks of one store
#pragma unroll
  for (int j = 0; j < TN; j += W) {
    const int p = p0 + out_of<O>(j, (lane >> 4) * 4);
    float bias[4 * W];
#pragma unroll
    for (int e = 0; e < 4 * W; ++e) bias[e] = a.h.bias && p + e < P ? a.h.bias[p + e] : 0.0f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int64_t n = n0 + i * 16 + (lane & 15);
      float y[4 * W];
#pragma unroll
      for (int e = 0; e < 4 * W; ++e) y[e] = acc[i][j + e / 4][e & 3] + bias[e];
      if (n < a.N && p < P) store_out<O, 4 * W>((O*)a.out + n * a.out_ld + p, y, P - p);
    }
  }
}

constexpr int kStepK = 64;  // columns of a step: 128 bytes of a row

// Where chunk c (16 bytes) of tile row r lies in LDS: rows of 128 bytes whose
// chunks are permuted, so that the 16 rows of an operand read fall on
// different banks.
template <class O, bool W>
__device__ __forceinline__ int swizzle(int row) {
  if constexpr (W && sizeof(O) == 2) return ((row >> 1) & 1) | (((row >> 3) & 3) << 1);
  return (row >> 1) & 7;
}

// BM rows and BN outputs per workgroup of WM x WN wavefronts.
template <class T, class O, int BM, int BN, int WM, int WN, bool ALIGNED>
__global__ void __launch_bounds__(64 * WM * WN) k_project(HeadArgs a, uint32_t row_tiles, uint32_t col_tiles) {
  constexpr int kWaves_ = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int kTile = (BM + BN) * 128;
  constexpr int kParts = (BM + BN) / 8 / kWaves_;  // groups of 8 rows per wavefront
  static_assert((BM / 8) % kWaves_ == 0 && (BN / 8) % kWaves_ == 0, "");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int D = a.h.D, P = a.h.P;
  const int64_t n0 = (int64_t)(blockIdx.x / col_tiles) * BM;
  const int p0 = (int)(blockIdx.x % col_tiles) * BN;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;

  // this lane's source rows: parts of BM rows of x, then of BN rows of W
  const T* src[kParts];
  int col[kParts];
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    const bool w = i * kWaves_ * 8 >= BM;
    const int row = (i * kWaves_ + wave) * 8 - (w ? BM : 0) + (lane >> 3);
    col[i] = ((lane & 7) ^ (w ? swizzle<O, true>(row) : swizzle<O, false>(row))) * 8;
    src[i] = w ? (const T*)a.h.weight + (int64_t)min(p0 + row, P - 1) * a.h.weight_ld
               : (const T*)a.x + min(n0 + row, a.N - 1) * a.x_ld;
  }
  auto stage = [&](int k0, char* to) {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      char* dst = to + (i * kWaves_ + wave) * 1024;
      const int k = k0 + col[i];
      if constexpr (ALIGNED) {
        const T* p = k < D ? src[i] + k : (const T*)&k_zeros;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                         (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
      } else {
        *(uint4*)(dst + lane * 16) = load8(src[i] + k, D - k);
      }
    }
  };

  f32x4 acc[TM][TN] = {};
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  int buf = 0;
  stage(0, lds);
  __syncthreads();
  for (int k0 = 0; k0 < D; k0 += kStepK, buf ^= 1) {
    if (k0 + kStepK < D) stage(k0 + kStepK, lds + (buf ^ 1) * kTile);
    const char* xs = lds + buf * kTile;
    const char* ws = xs + BM * 128;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int c = ks * 4 + (lane >> 4);
      uint4 w[TN], x[TM];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = wn + out_of<O>(j, lane & 15);
        w[j] = *(const uint4*)(ws + r * 128 + ((c ^ swizzle<O, true>(r)) << 4));
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int r = wm + i * 16 + (lane & 15);
        x[i] = *(const uint4*)(xs + r * 128 + ((c ^ swizzle<O, false>(r)) << 4));
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma16(w[j], x[i], acc[i][j], T{});
    }
    __syncthreads();
  }
  finish_tile<T, O>(a, n0 + wm, p0 + wn, acc);
}

template <class T, class O, int BM, int BN, int WM, int WN, bool ALIGNED>
void launch_tiles(const HeadArgs& a, hipStream_t s) {
  const uint32_t rows = (uint32_t)((a.N + BM - 1) / BM), cols = ((uint32_t)a.h.P + BN - 1) / BN;
  auto* k = k_project<T, O, BM, BN, WM, WN, ALIGNED>;
  constexpr int bytes = 2 * (BM + BN) * 128;
  if (bytes > 65536) (void)hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  hipLaunchKernelGGL(k, dim3(rows * cols), dim3(64 * WM * WN), bytes, s, a, rows, cols);
}

template <class T, class O>
void launch_project(HeadArgs a, hipStream_t s) {
  if (a.adapter) {
    constexpr int terms = kTerms<T, O>;
    a.uk = terms * a.rp;
    hipLaunchKernelGGL((k_low_row<T, terms>), dim3((uint32_t)a.N), dim3(256), 0, s, a);
  }
  const bool aligned = a.h.D % 8 == 0 && a.x_ld % 8 == 0 && a.h.weight_ld % 8 == 0 && !((uintptr_t)a.x & 15) &&
                       !((uintptr_t)a.h.weight & 15);
  const auto tiles = [&](int64_t m, int64_t n) { return ((a.N + m - 1) / m) * ((a.h.P + n - 1) / n); };
  if (!aligned)
    launch_tiles<T, O, 64, 64, 2, 2, false>(a, s);
  else if (tiles(256, 256) >= 256)
    launch_tiles<T, O, 256, 256, 2, 4, true>(a, s);
  else if (tiles(128, 128) >= 256)
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

// Workspace: the terms of u (at most three), then the rows' powers of two.
static int padded_rank(const wd_head* h) { return (h->rank + 7) / 8 * 8; }
static size_t u_bytes(const wd_head* h, int64_t N) { return align_up((uint64_t)N * 3 * padded_rank(h) * 2, 256); }
static size_t project_bytes(const wd_head* h, int64_t N) {
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
  HeadArgs a{*h, x, x_ld, N, adapter, out, out_ld, (uint16_t*)ws,
             adapter ? (float*)((char*)ws + u_bytes(h, N)) : nullptr, adapter ? padded_rank(h) : 0, 0};
  hipStream_t s = (hipStream_t)stream;
  if (h->type == WD_F16)
    out_type == WD_F32 ? launch_project<Half, F32>(a, s) : launch_project<Half, Half>(a, s);
  else
    out_type == WD_F32 ? launch_project<Bf16, F32>(a, s) : launch_project<Bf16, Bf16>(a, s);
  return hip_check(hipGetLastError(), "project");
}
