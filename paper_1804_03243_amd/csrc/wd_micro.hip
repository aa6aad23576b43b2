// Matrices in microscaled 4-bit floating point, and their product.
//
// A row's values in blocks of 32: a block has a power of two 2^(s - 127), s one byte,
// and a value is 0, 0.5, 1, 1.5, 2, 3, 4 or 6 times it with a sign, four bits
// (sign, two of exponent, one of mantissa).  s = floor(log2 of the block's largest
// magnitude) + 125, at least 0; values round to nearest, ties to the even code,
// magnitudes above 6 to 6.  s = 255 says that the block is not a number, which a block
// with an infinity or NaN becomes as a whole.
//
// In memory a row is ceil(D / 32) blocks of 16 bytes, the lower four bits first, and
// 16 ceil(D / 512) bytes of scales: the matrix instruction takes 128 columns, 32 of
// them in a quarter of the wavefront, with a scale byte chosen from a register by a constant;
// so the scales of 512 columns stand as [quarter q][product h], block 4 h + q at 4 q + h.
// Columns past D are zeros, scales past the last block 0.
#include <algorithm>

#include "wd_host.h"
#include "wd_tile.h"

namespace wd {

__device__ __host__ __forceinline__ int64_t micro_blocks(int64_t D) { return (D + 31) / 32; }
__device__ __host__ __forceinline__ int64_t micro_scales(int64_t D) { return (D + 511) / 512 * 16; }

// Where the scale of block b of a row stands.
__device__ __forceinline__ int64_t scale_at(int64_t b) { return (b & ~15ll) + (b & 3) * 4 + ((b >> 2) & 3); }

// Four lanes to a block, eight values each.  Bound by memory.  Lanes of a scale row's
// padding write its zeros.
template <class T>
__global__ void __launch_bounds__(256) k_micro(const T* x, int64_t ld, int64_t N, int D, uint32_t* codes, uint8_t* scales) {
  const int64_t blocks = micro_blocks(D), sl = micro_scales(D), per = sl * 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * per; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / per;
    const int e = (int)(i % per), k = e * 8;  // (per is a multiple of 64: a block's lanes stay together)
    float v[8] = {};
    if (k + 8 <= D) {
      const Few<T, 8> w = *(const Few<T, 8>*)(x + n * ld + k);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = w.v[j].f();
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (k + j < D) v[j] = x[n * ld + k + j].f();
    }
    uint32_t top = 0;  // magnitudes order as their bits do
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const bool bad = top >= 0x7f800000u;
    const int s = max((int)(top >> 23) - 2, 0);
    const float by = __uint_as_float((uint32_t)(254 - s) << 23);  // 2^(127 - s), exact
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * by, v[1] * by, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * by, v[3] * by, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * by, v[5] * by, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * by, v[7] * by, 1.0f, 3);
    if (e < blocks * 4) codes[n * blocks * 4 + e] = bad ? 0 : c;
    if ((e & 3) == 0) scales[n * sl + scale_at(e >> 2)] = e >= blocks * 4 ? 0 : bad ? 255 : (uint8_t)s;
  }
}

// The values, exact in bfloat16 and 32 bits.
template <class O>
__global__ void __launch_bounds__(256) k_micro_values(const uint32_t* codes, const uint8_t* scales, int64_t N, int D, O* out, int64_t ld) {
  const int64_t blocks = micro_blocks(D), sl = micro_scales(D), per = (D + 7) / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * per; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / per;
    const int e = (int)(i % per);
    const uint32_t c = codes[n * blocks * 4 + e];
    const uint32_t s = scales[n * sl + scale_at(e >> 2)];
    const float unit = s == 255 ? NAN : s == 0 ? 0x1p-127f : __uint_as_float(s << 23);
    Few<O, 8> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = c >> (4 * j), m = b & 7;
      const float q = m < 2 ? 0.5f * m : (float)((2 | (m & 1)) << (m >> 1)) * 0.25f;
      v.v[j] = O::of((b & 8 ? -q : q) * unit);
    }
    store_out(out + n * ld + e * 8, v, D - e * 8);
  }
}

typedef __attribute__((ext_vector_type(8))) int i32x8;

// 128 columns of 16 rows by 16: the scales' byte H of each register.
template <int H>
__device__ __forceinline__ f32x4 mfma4(uint4 a, uint4 b, f32x4 c, int sa, int sb) {
  const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, H, sa, H, sb);
}

struct MicroArgs {
  const uint8_t *x, *xs, *w, *ws;  // codes and scales of rows and weights
  int64_t N;
  int32_t P, blocks, sl;           // blocks and scale bytes of a row
  const float* bias;
  void* out;
  int64_t out_ld;
};

// A wavefront per 16 outputs and 16 rows, operands straight from memory: the simplest product.
template <class O>
__global__ void __launch_bounds__(256) k_micro_product(MicroArgs a, uint32_t col_blocks) {
  const int lane = threadIdx.x & 63, l = lane & 15, quad = lane >> 4;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t n = at / col_blocks * 16 + l;
  const int p = (int)(at % col_blocks) * 16;
  if (n - l >= a.N) return;
  const int64_t wr = min(p + l, a.P - 1), xr = min<int64_t>(n, a.N - 1);
  f32x4 acc = {0, 0, 0, 0};
  for (int b = 0; b < a.blocks; b += 16) {
    const int sw = *(const int*)(a.ws + wr * a.sl + b + quad * 4), sx = *(const int*)(a.xs + xr * a.sl + b + quad * 4);
    uint4 w[4], x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int k = b + h * 4 + quad;
      w[h] = x[h] = make_uint4(0, 0, 0, 0);
      if (k < a.blocks) w[h] = *(const uint4*)(a.w + (wr * a.blocks + k) * 16), x[h] = *(const uint4*)(a.x + (xr * a.blocks + k) * 16);
    }
    acc = mfma4<0>(w[0], x[0], acc, sw, sx);
    acc = mfma4<1>(w[1], x[1], acc, sw, sx);
    acc = mfma4<2>(w[2], x[2], acc, sw, sx);
    acc = mfma4<3>(w[3], x[3], acc, sw, sx);
  }
  if (n >= a.N) return;
  Few<O, 4> v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v.v[e] = O::of(acc[e] + (a.bias ? a.bias[min(p + quad * 4 + e, a.P - 1)] : 0.0f));
  store_out((O*)a.out + n * a.out_ld + p + quad * 4, v, a.P - p - quad * 4);
}

template <class T>
static void launch_micro(const void* x, int64_t ld, int64_t N, int D, void* codes, void* scales, hipStream_t s) {
  const uint64_t blocks = ((uint64_t)N * micro_scales(D) * 4 + 255) / 256;
  hipLaunchKernelGGL((k_micro<T>), dim3((uint32_t)std::min<uint64_t>(blocks, 1 << 16)), dim3(256), 0, s, (const T*)x, ld, N, D, (uint32_t*)codes,
                     (uint8_t*)scales);
}

static void quantize(const void* x, int64_t ld, int64_t N, int D, int32_t type, void* codes, void* scales, hipStream_t s) {
  if (type == WD_F32)
    launch_micro<F32>(x, ld, N, D, codes, scales, s);
  else if (type == WD_F16)
    launch_micro<Half>(x, ld, N, D, codes, scales, s);
  else
    launch_micro<Bf16>(x, ld, N, D, codes, scales, s);
}

template <class O>
static void launch_micro_product(const MicroArgs& a, hipStream_t s) {
  const uint32_t cols = ((uint32_t)a.P + 15) / 16;
  const uint64_t waves = (uint64_t)((a.N + 15) / 16) * cols;
  hipLaunchKernelGGL((k_micro_product<O>), dim3((uint32_t)((waves + 3) / 4)), dim3(256), 0, s, a, cols);
}

}  // namespace wd

using namespace wd;

static wd_status check_micro(const wd_micro* m, const char* what) {
  if (!m) return fail(WD_EINVAL, std::string(what) + ": null matrix");
  if (m->rows < 0 || m->rows > INT32_MAX) return fail(WD_EINVAL, std::string(what) + ": rows out of range");
  if (m->D < 1 || m->D >= (1 << 22)) return fail(WD_EINVAL, std::string(what) + ": D out of range");
  if (m->rows > 0 && (!m->codes || !m->scales)) return fail(WD_EINVAL, std::string(what) + ": null codes or scales");
  if ((uintptr_t)m->codes & 15 || (uintptr_t)m->scales & 15) return fail(WD_EINVAL, std::string(what) + ": codes and scales must be 16-byte aligned");
  return WD_OK;
}

extern "C" wd_status wd_micro_bytes(int64_t rows, int32_t D, size_t* codes, size_t* scales) {
  if (!codes || !scales) return fail(WD_EINVAL, "micro_bytes: null output");
  if (rows < 0 || rows > INT32_MAX) return fail(WD_EINVAL, "micro_bytes: rows out of range");
  if (D < 1 || D >= (1 << 22)) return fail(WD_EINVAL, "micro_bytes: D out of range");
  *codes = (size_t)rows * micro_blocks(D) * 16;
  *scales = (size_t)rows * micro_scales(D);
  return WD_OK;
}

extern "C" wd_status wd_micro_quantize(const void* x, int32_t type, int64_t x_ld, const wd_micro* out, void* stream) {
  wd_status st = check_micro(out, "micro_quantize");
  if (st != WD_OK) return st;
  if (type != WD_F32 && type != WD_F16 && type != WD_BF16) return fail(WD_EINVAL, "micro_quantize: unknown type");
  if (x_ld < out->D) return fail(WD_EINVAL, "micro_quantize: row stride too small");
  if (out->rows == 0) return WD_OK;
  if (!x) return fail(WD_EINVAL, "micro_quantize: null rows");
  if ((uintptr_t)x & (type == WD_F32 ? 3 : 1)) return fail(WD_EINVAL, "micro_quantize: misaligned rows");
  quantize(x, x_ld, out->rows, out->D, type, (void*)out->codes, (void*)out->scales, (hipStream_t)stream);
  return hip_check(hipGetLastError(), "micro_quantize");
}

extern "C" wd_status wd_micro_values(const wd_micro* m, void* out, int32_t type, int64_t out_ld, void* stream) {
  wd_status st = check_micro(m, "micro_values");
  if (st != WD_OK) return st;
  if (type != WD_F32 && type != WD_BF16) return fail(WD_EINVAL, "micro_values: type must be WD_F32 or WD_BF16");
  if (out_ld < m->D) return fail(WD_EINVAL, "micro_values: row stride too small");
  if (m->rows == 0) return WD_OK;
  if (!out) return fail(WD_EINVAL, "micro_values: null output");
  if ((uintptr_t)out & (type == WD_F32 ? 3 : 1)) return fail(WD_EINVAL, "micro_values: misaligned output");
  const uint64_t blocks = ((uint64_t)m->rows * ((m->D + 7) / 8) + 255) / 256;
  const dim3 grid((uint32_t)std::min<uint64_t>(blocks, 1 << 16)), block(256);
  hipStream_t s = (hipStream_t)stream;
  if (type == WD_F32)
    hipLaunchKernelGGL((k_micro_values<F32>), grid, block, 0, s, (const uint32_t*)m->codes, (const uint8_t*)m->scales, m->rows, m->D, (F32*)out, out_ld);
  else
    hipLaunchKernelGGL((k_micro_values<Bf16>), grid, block, 0, s, (const uint32_t*)m->codes, (const uint8_t*)m->scales, m->rows, m->D, (Bf16*)out, out_ld);
  return hip_check(hipGetLastError(), "micro_values");
}

constexpr int64_t kMicroRows = 1 << 20;  // rows of a launch

static wd_status micro_project_bytes(const wd_micro* w, int64_t N, size_t* bytes) {
  wd_status st = check_micro(w, "micro_project");
  if (st != WD_OK) return st;
  if (w->rows < 1 || w->rows >= (1 << 24)) return fail(WD_EINVAL, "micro_project: outputs out of range");
  if (N < 0 || N > INT32_MAX) return fail(WD_EINVAL, "micro_project: N out of range");
  const int64_t n = std::min(N, kMicroRows);
  *bytes = align_up((uint64_t)n * micro_blocks(w->D) * 16, 256) + align_up((uint64_t)n * micro_scales(w->D), 256);
  return WD_OK;
}

extern "C" wd_status wd_micro_project_workspace_bytes(const wd_micro* w, int64_t N, size_t* bytes) {
  if (!bytes) return fail(WD_EINVAL, "micro_project_workspace_bytes: null output");
  return micro_project_bytes(w, N, bytes);
}

extern "C" wd_status wd_micro_project(const wd_micro* w, const float* bias, const void* x, int32_t type, int64_t x_ld, int64_t N, void* out,
                                      int32_t out_type, int64_t out_ld, void* ws, size_t ws_bytes, void* stream) {
  size_t need = 0;
  wd_status st = micro_project_bytes(w, N, &need);
  if (st != WD_OK) return st;
  if (type != WD_F32 && type != WD_F16 && type != WD_BF16) return fail(WD_EINVAL, "micro_project: unknown type");
  if (out_type != WD_F32 && out_type != WD_F16 && out_type != WD_BF16) return fail(WD_EINVAL, "micro_project: unknown out_type");
  if (x_ld < w->D || out_ld < w->rows) return fail(WD_EINVAL, "micro_project: row stride too small");
  if (N == 0) return WD_OK;
  if (!x || !out) return fail(WD_EINVAL, "micro_project: null rows or output");
  if ((uintptr_t)x & (type == WD_F32 ? 3 : 1) || (uintptr_t)out & (out_type == WD_F32 ? 3 : 1) || (uintptr_t)bias & 3)
    return fail(WD_EINVAL, "micro_project: misaligned array");
  if (!ws || ws_bytes < need || (uintptr_t)ws & 255) return fail(WD_EINVAL, "micro_project: workspace missing, too small or not 256-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  const size_t xe = type == WD_F32 ? 4 : 2, oe = out_type == WD_F32 ? 4 : 2;
  // (a launch has fewer than 2^32 threads)
  const int64_t most = std::max<int64_t>(16, std::min<int64_t>(kMicroRows, (1ll << 24) / ((w->rows + 15) / 16) * 16));
  for (int64_t n0 = 0; n0 < N; n0 += most) {
    const int64_t n = std::min(most, N - n0);
    uint8_t *codes = (uint8_t*)ws, *scales = codes + align_up((uint64_t)n * micro_blocks(w->D) * 16, 256);
    quantize((const char*)x + n0 * x_ld * xe, x_ld, n, w->D, type, codes, scales, s);
    MicroArgs a{codes, scales, (const uint8_t*)w->codes, (const uint8_t*)w->scales, n, (int32_t)w->rows, (int32_t)micro_blocks(w->D), (int32_t)micro_scales(w->D),
                bias, (char*)out + n0 * out_ld * oe, out_ld};
    if (out_type == WD_F32)
      launch_micro_product<F32>(a, s);
    else if (out_type == WD_F16)
      launch_micro_product<Half>(a, s);
    else
      launch_micro_product<Bf16>(a, s);
  }
  return hip_check(hipGetLastError(), "micro_project");
}
