// The output layer with low-rank adapters: out[n] = W x[n] + b + s_g B_g (A_g x[n]).
//
// Two launches: u[n] = s_g A_g x[n] (k_low, 32-bit sums), then the shared
// product in tiles of matrix instructions with the adapters' part, the bias and
// the rounding to the output's type added as a tile is stored (k_project).
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
  const int32_t* adapter;
  void* out;
  int64_t out_ld;
  float* u;  // [N][R]
};

__device__ __forceinline__ int adapter_of(const HeadArgs& a, int64_t n) {
  if (!a.adapter || a.h.n_adapters == 0) return -1;
  const int g = a.adapter[n];
  return g >= 0 && g < a.h.n_adapters ? g : -1;
}

// u[n][r]: a wavefront per row, the ranks one after another.
template <class T>
__global__ void __launch_bounds__(256) k_low(HeadArgs a) {
  const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= a.N) return;
  const int g = adapter_of(a, n), D = a.h.D, R = a.h.rank;
  if (g < 0) return;  // (never read)
  const T* x = (const T*)a.x + n * a.x_ld;
  const float sc = a.h.scale ? a.h.scale[g] : 1.0f;
  for (int r = 0; r < R; ++r) {
    const T* w = (const T*)a.h.a + ((int64_t)g * R + r) * D;
    float s = 0.0f;
    for (int k = lane_id(); k < D; k += 64) s = fmaf(x[k].f(), w[k].f(), s);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane_id() == 0) a.u[n * R + r] = s * sc;
  }
}

// A tile of 64 rows and 64 outputs per workgroup, 32 x 32 per wavefront.
template <class T, class O>
__global__ void __launch_bounds__(256) k_project(HeadArgs a, uint32_t col_tiles) {
  constexpr int kRow = 40;  // 32 values and 8 of padding
  __shared__ __attribute__((aligned(16))) T xs[64 * kRow], ws[64 * kRow];
  const int D = a.h.D, P = a.h.P;
  const int64_t n0 = (int64_t)(blockIdx.x / col_tiles) * 64;
  const int p0 = (int)(blockIdx.x % col_tiles) * 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
  f32x4 acc[2][2] = {};
  const int lr = threadIdx.x >> 2, lk = (threadIdx.x & 3) * 8;  // this thread's row and columns of a tile
  for (int k0 = 0; k0 < D; k0 += 32) {
    const T* x = (const T*)a.x + (n0 + lr) * a.x_ld;
    const T* w = (const T*)a.h.weight + (int64_t)(p0 + lr) * a.h.weight_ld;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = k0 + lk + i;
      xs[lr * kRow + lk + i] = n0 + lr < a.N && k < D ? x[k] : T{0};
      ws[lr * kRow + lk + i] = p0 + lr < P && k < D ? w[k] : T{0};
    }
    __syncthreads();
    uint4 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = *(const uint4*)&xs[(wm + i * 16 + (lane & 15)) * kRow + (lane >> 4) * 8];
      fb[i] = *(const uint4*)&ws[(wn + i * 16 + (lane & 15)) * kRow + (lane >> 4) * 8];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = mfma16(fa[i], fb[j], acc[i][j], T{});
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t n = n0 + wm + i * 16 + (lane >> 4) * 4 + e;
      if (n >= a.N) continue;
      const int g = adapter_of(a, n), R = a.h.rank;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int p = p0 + wn + j * 16 + (lane & 15);
        if (p >= P) continue;
        float y = acc[i][j][e] + (a.h.bias ? a.h.bias[p] : 0.0f);
        if (g >= 0) {
          const T* b = (const T*)a.h.b + ((int64_t)g * P + p) * R;
          float low = 0.0f;
          for (int r = 0; r < R; ++r) low = fmaf(a.u[n * R + r], b[r].f(), low);
          y += low;
        }
        ((O*)a.out)[n * a.out_ld + p] = O::of(y);
      }
    }
}

template <class T>
void launch_project(const HeadArgs& a, int32_t out_type, hipStream_t s) {
  if (a.adapter && a.h.n_adapters)
    hipLaunchKernelGGL(k_low<T>, dim3((uint32_t)((a.N + 3) / 4)), dim3(256), 0, s, a);
  const uint32_t cols = ((uint32_t)a.h.P + 63) / 64;
  const dim3 grid((uint32_t)((a.N + 63) / 64) * cols);
  if (out_type == WD_F32)
    hipLaunchKernelGGL((k_project<T, F32>), grid, dim3(256), 0, s, a, cols);
  else
    hipLaunchKernelGGL((k_project<T, T>), grid, dim3(256), 0, s, a, cols);
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

static size_t project_bytes(const wd_head* h, int64_t N) {
  return h->n_adapters > 0 ? align_up((uint64_t)N * h->rank * sizeof(float), 256) : 0;
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
  const size_t need = adapter ? project_bytes(h, N) : 0;
  if (need && (!ws || ws_bytes < need || (uintptr_t)ws & 255))
    return fail(WD_EINVAL, "project: workspace missing, too small or not 256-byte aligned");
  if (((uint64_t)N + 63) / 64 * (((uint64_t)h->P + 63) / 64) > INT32_MAX)
    return fail(WD_EINVAL, "project: too many rows for one call");
  HeadArgs a{*h, x, x_ld, N, adapter, out, out_ld, (float*)ws};
  if (h->type == WD_F16)
    launch_project<Half>(a, out_type, (hipStream_t)stream);
  else
    launch_project<Bf16>(a, out_type, (hipStream_t)stream);
  return hip_check(hipGetLastError(), "project");
}
