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
#include <type_traits>

#include "wd_host.h"
#include "wd_tile.h"

namespace wd {

__device__ __host__ __forceinline__ int64_t micro_blocks(int64_t D) { return (D + 31) / 32; }
__device__ __host__ __forceinline__ int64_t micro_scales(int64_t D) { return (D + 511) / 512 * 16; }

// Where the scale of block b of a row stands.
__device__ __forceinline__ int64_t scale_at(int64_t b) { return (b & ~15ll) + (b & 3) * 4 + ((b >> 2) & 3); }

// Eight values of a row of D from column k on, zeros past its end.
template <class T>
__device__ __forceinline__ void load_values(const T* x, int k, int D, float (&v)[8]) {
  if (k + 8 <= D) {
    const Few<T, 8> w = *(const Few<T, 8>*)(x + k);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = w.v[j].f();
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < D ? x[k + j].f() : 0.0f;
  }
}

// A lane's eight values as codes; the four lanes of a block, side by side, hold its 32.
// Returns the block's scale byte.
__device__ __forceinline__ uint32_t to_codes(const float (&v)[8], uint32_t& codes) {
  uint32_t top = 0;  // magnitudes order as their bits do
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, dpp32<kDppQuadSwap1>(top, 0));
  top = max(top, dpp32<kDppQuadSwap2>(top, 0));
  const bool bad = top >= 0x7f800000u;
  const int s = max((int)(top >> 23) - 2, 0);
  const float by = __uint_as_float((uint32_t)(254 - s) << 23);  // 2^(127 - s), exact
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * by, v[1] * by, 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * by, v[3] * by, 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * by, v[5] * by, 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * by, v[7] * by, 1.0f, 3);
  codes = bad ? 0 : c;
  return bad ? 255 : (uint32_t)s;
}

// Four lanes to a block, eight values each.  Bound by memory: 100000 rows of 1024 in bfloat16 51
// us, 5.1 TB/s.  Lanes of a scale row's padding write its zeros.
template <class T>
__global__ void __launch_bounds__(256) k_micro(const T* x, int64_t ld, uint32_t N, int D, uint32_t* codes, uint8_t* scales) {
  const int64_t blocks = micro_blocks(D), sl = micro_scales(D);
  const uint32_t per = (uint32_t)sl * 4;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < N * per; i += gridDim.x * 256) {
    const int64_t n = i / per;
    const int e = (int)(i % per), k = e * 8;  // (per is a multiple of 64: a block's lanes stay together)
    float v[8];
    load_values(x + n * ld, k, D, v);
    uint32_t c;
    const uint32_t s = to_codes(v, c);
    if (e < blocks * 4) codes[n * blocks * 4 + e] = c;
    if ((e & 3) == 0) scales[n * sl + scale_at(e >> 2)] = e >= blocks * 4 ? 0 : (uint8_t)s;
  }
}

// The values, exact in bfloat16 and 32 bits.  Bound by memory: 100000 rows of 1024 to bfloat16 63
// us, 4.1 TB/s.
template <class O>
__global__ void __launch_bounds__(256) k_micro_values(const uint32_t* codes, const uint8_t* scales, uint32_t N, int D, O* out, int64_t ld) {
  const int64_t blocks = micro_blocks(D), sl = micro_scales(D);
  const uint32_t per = (D + 7) / 8;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < N * per; i += gridDim.x * 256) {
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
  bool stream;                     // outputs past the caches
};

// Many rows: tiles of BM rows and BN outputs, as the 16-bit products go (Tile): a step is
// 128 bytes of a row, here 256 columns, its halves 128.  The scales of two steps
// come with the even one, 16 bytes of each row, into two places of their own.  64000 rows of 1024 to
// 6000 outputs in 32 bits 390 us: bound by the outputs' 1.5 GB (300 us), which tiles of three workgroups
// on a compute unit write while others multiply (in tiles of 256 x 256 837 us, of 256 x 128 526, 64-row
// tiles of eight wavefronts 446).
template <class O, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_micro_tiles(MicroArgs a, uint32_t row_tiles, uint32_t col_tiles) {
  constexpr int kWaves_ = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  using X = Side<BM, false, kWaves_>;
  using W = Side<BN, false, kWaves_>;
  constexpr int kStep = (BM + BN) * 128, kScales = 2 * kStep, kScaleStep = (BM + BN) * 16;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  uint32_t row_tile, col_tile;
  my_tile(row_tiles, col_tiles, row_tile, col_tile);
  const int64_t n0 = (int64_t)row_tile * BM;
  const int p0 = (int)col_tile * BN;
  const int wave = wave_number(), lane = threadIdx.x & 63, l = lane & 15, quad = lane >> 4;
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int64_t ld = (int64_t)a.blocks * 16;
  const int rows = (int)min<int64_t>(BM, a.N - n0), outs = min(BN, a.P - p0), K = a.blocks * 8;
  X x;
  W w;
  x.init({a.x + n0 * ld, ld, rows}, wm, lds0);
  w.init({a.w + (int64_t)p0 * ld, ld, outs}, wn, lds0 + X::kBytes);
  // (64 rows' scales to a load, the tile's rows and then its outputs)
  const int scale_row = wave * 64 + lane;
  const uint32_t scale_from = (uint32_t)((scale_row < BM ? min(scale_row, rows - 1) : min(scale_row - BM, outs - 1)) * a.sl);
  const auto stage = [&](int k0, int at) {
    if (k0 / kStepK % 2 == 0) {
      const uint32_t to = lds0 + kScales + (k0 / kStepK / 2 & 1) * kScaleStep + wave * 1024;
      if (scale_row < BM)
        load_to_lds(a.xs + n0 * a.sl + k0 / kStepK / 2 * 16, scale_from, to);
      else if (scale_row < BM + BN)
        load_to_lds(a.ws + (int64_t)p0 * a.sl + k0 / kStepK / 2 * 16, scale_from, to);
    }
    x.stage(k0, K, at);
    w.stage(k0, K, at);
  };
  struct Operands {
    uint4 w[TN], x[TM];
  } even, odd;
  struct Scales {  // of a step: byte 0 its first half's, byte 1 its second's
    int w[TN], x[TM];
  } scale, next_scale;
  const auto read = [&](int at, int half, Operands& o) {
#pragma unroll
    for (int j = 0; j < TN; ++j) o.w[j] = w.rows(at, j, half);
#pragma unroll
    for (int i = 0; i < TM; ++i) o.x[i] = x.rows(at, i, half);
  };
  const auto read_scales = [&](int k0, Scales& s) {
    const char* from = lds + kScales + (k0 / kStepK / 2 & 1) * kScaleStep + (wm + l) * 16 + quad * 4;
    const int by = k0 / kStepK % 2 * 16;
#pragma unroll
    for (int j = 0; j < TN; ++j) s.w[j] = *(const int*)(from + (BM + wn - wm + j * 16) * 16) >> by;
#pragma unroll
    for (int i = 0; i < TM; ++i) s.x[i] = *(const int*)(from + i * 256) >> by;
  };
  // (read from memory at the tile's end it would be a round trip that nothing hides)
  float* kept_bias = (float*)(lds + 2 * (kStep + kScaleStep));
  static_assert(BN <= 64 * kWaves_, "");
  const float my_bias = a.bias && (int)threadIdx.x < min(BN, outs) ? a.bias[p0 + threadIdx.x] : 0.0f;
  f32x4 acc[TM][TN] = {};
  const auto products = [&](const Operands& o, auto half) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma4<half.value>(o.w[j], o.x[i], acc[i][j], scale.w[j], scale.x[i]);
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1 + half.value, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, TM * TN / (TM + TN), 0);
    }
  };
  int now = 0, next = kStep;
  stage(0, now);
  if (kStepK < K) stage(kStepK, next);
  loads_left<0>();
  __syncthreads();
  read(now, 0, even);
  read_scales(0, scale);
  for (int k0 = 0; k0 < K; k0 += kStepK) {
    read(now, 1, odd);
    products(even, std::integral_constant<int, 0>{});
    loads_left<0>();
    __syncthreads();  // this step has been read, the next one is there
    if (k0 + 2 * kStepK < K) stage(k0 + 2 * kStepK, now);
    read(next, 0, even);
    read_scales(k0 + kStepK, next_scale);
    products(odd, std::integral_constant<int, 1>{});
    scale = next_scale;
    now = next;
    next = kStep - next;
  }
  if ((int)threadIdx.x < BN) kept_bias[threadIdx.x] = my_bias;
  __syncthreads();  // (every wavefront has read its last operands)
  f32x4 bias[TN];
#pragma unroll
  for (int j = 0; j < TN; ++j) bias[j] = *(const f32x4*)(kept_bias + wn + j * 16 + quad * 4);
  store_tile<O, TM, TN>((O*)a.out + (n0 + wm) * a.out_ld + p0 + wn, a.out_ld, a.N - n0 - wm, a.P - p0 - wn, lds + wave * kStoreBytes<O, TN>,
                        [&](int i, int j, int e) { return acc[i][j][e] + bias[j][e]; }, a.stream);
}

// A few rows (kFewRows at most) in one launch: every workgroup brings them to their four-bit
// form itself, in LDS, while its first reads of W are under way.  A wavefront takes 16
// outputs, W straight from memory, the next 512 columns' reads under way while one is
// multiplied.  Rows in LDS are an odd number of 16-byte blocks apart, so that reads of
// several rows fall on different banks.  (Rows of 1024 to 6000 outputs this way and in two launches:
// 1 row 3.5 and 5.4 us, 8 rows 4.8 and 6.0, 16 rows 6.3 and 5.9; 8 rows of 2000 to 5000 7.9 and 7.4.)
constexpr int kFewRows = 8;
template <class T, class O>
__global__ void __launch_bounds__(256, 4) k_micro_few(MicroArgs a, const T* rows, int64_t ld, int D) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l = lane & 15, quad = lane >> 4;
  const int p0 = (blockIdx.x * 4 + wave) * 16, N = (int)a.N;
  const int line = a.blocks | 1;
  uint8_t* scales = (uint8_t*)lds + N * line * 16;
  const int64_t r = min(p0 + l, a.P - 1);
  struct Operands {
    uint4 w[4];
    int s;
  } o[2];
  const auto read = [&](int b, Operands& o) {
    o.s = *(const int*)(a.ws + r * a.sl + b + quad * 4);
#pragma unroll
    for (int h = 0; h < 4; ++h) o.w[h] = *(const uint4*)(a.w + (r * a.blocks + min(b + h * 4 + quad, a.blocks - 1)) * 16);
  };
  read(0, o[0]);
  const int per = a.sl * 4;  // (a multiple of 64: a block's lanes stay together)
  for (int i = threadIdx.x; i < N * per; i += 256) {
    const int n = i / per, e = i % per;
    float v[8];
    load_values(rows + n * ld, e * 8, D, v);
    uint32_t c;
    const uint32_t s = to_codes(v, c);
    if (e < a.blocks * 4) *(uint32_t*)(lds + n * line * 16 + e * 4) = c;
    if ((e & 3) == 0) scales[n * a.sl + scale_at(e >> 2)] = e >= a.blocks * 4 ? 0 : (uint8_t)s;
  }
  __syncthreads();
  f32x4 acc = {0, 0, 0, 0};
  const int n = min(l, N - 1);  // (the other lanes' products are of no use)
  const auto multiply = [&](int b, const Operands& o) {
    const int s = *(const int*)(scales + n * a.sl + b + quad * 4);
    uint4 x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int k = b + h * 4 + quad;
      x[h] = *(const uint4*)(lds + (n * line + min(k, a.blocks - 1)) * 16);
      if (k >= a.blocks) x[h] = make_uint4(0, 0, 0, 0);
    }
    acc = mfma4<0>(o.w[0], x[0], acc, o.s, s);
    acc = mfma4<1>(o.w[1], x[1], acc, o.s, s);
    acc = mfma4<2>(o.w[2], x[2], acc, o.s, s);
    acc = mfma4<3>(o.w[3], x[3], acc, o.s, s);
  };
  for (int b = 0; b < a.blocks; b += 32) {
    if (b + 16 < a.blocks) read(b + 16, o[1]);
    multiply(b, o[0]);
    if (b + 32 < a.blocks) read(b + 32, o[0]);
    if (b + 16 < a.blocks) multiply(b + 16, o[1]);
  }
  const int p = p0 + quad * 4;
  if (l >= N) return;
  Few<O, 4> v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v.v[e] = O::of(acc[e] + (a.bias ? a.bias[min(p + e, a.P - 1)] : 0.0f));
  store_out((O*)a.out + l * a.out_ld + p, v, a.P - p);
}

// Rows of a launch, whose lanes are counted in 32 bits.
static int64_t micro_rows(int64_t lanes_of_a_row) { return std::max<int64_t>(1, (1 << 30) / lanes_of_a_row); }

template <class T>
static void launch_micro(const void* x, int64_t ld, int64_t N, int D, void* codes, void* scales, hipStream_t s) {
  const int64_t per = micro_scales(D) * 4, most = micro_rows(per);
  for (int64_t n0 = 0; n0 < N; n0 += most) {
    const int64_t n = std::min(most, N - n0);
    hipLaunchKernelGGL((k_micro<T>), dim3((uint32_t)std::min<int64_t>((n * per + 255) / 256, 1 << 16)), dim3(256), 0, s, (const T*)x + n0 * ld, ld,
                       (uint32_t)n, D, (uint32_t*)codes + n0 * micro_blocks(D) * 4, (uint8_t*)scales + n0 * micro_scales(D));
  }
}

template <class O>
static void launch_values(const wd_micro* m, void* out, int64_t ld, hipStream_t s) {
  const int64_t per = (m->D + 7) / 8, most = micro_rows(per);
  for (int64_t n0 = 0; n0 < m->rows; n0 += most) {
    const int64_t n = std::min(most, m->rows - n0);
    hipLaunchKernelGGL((k_micro_values<O>), dim3((uint32_t)std::min<int64_t>((n * per + 255) / 256, 1 << 16)), dim3(256), 0, s,
                       (const uint32_t*)m->codes + n0 * micro_blocks(m->D) * 4, (const uint8_t*)m->scales + n0 * micro_scales(m->D), (uint32_t)n, m->D,
                       (O*)out + n0 * ld, ld);
  }
}

static void quantize(const void* x, int64_t ld, int64_t N, int D, int32_t type, void* codes, void* scales, hipStream_t s) {
  if (type == WD_F32)
    launch_micro<F32>(x, ld, N, D, codes, scales, s);
  else if (type == WD_F16)
    launch_micro<Half>(x, ld, N, D, codes, scales, s);
  else
    launch_micro<Bf16>(x, ld, N, D, codes, scales, s);
}

template <class O, int BM, int BN, int WM, int WN>
static void launch_micro_tiles(const MicroArgs& a, hipStream_t s) {
  const uint32_t rows = (uint32_t)((a.N + BM - 1) / BM), cols = ((uint32_t)a.P + BN - 1) / BN;
  auto* k = k_micro_tiles<O, BM, BN, WM, WN>;
  constexpr int stages = 2 * (BM + BN) * (128 + 16), bytes = stages + BN * 4;
  static_assert(kStoreBytes<O, BN / WN / 16> * WM * WN <= stages, "");
  static std::atomic<uint64_t> done{0};
  allow_lds((const void*)k, bytes, done);
  hipLaunchKernelGGL(k, dim3(rows * cols), dim3(64 * WM * WN), bytes, s, a, rows, cols);
}

template <class T, class O>
static void launch_micro_few(const MicroArgs& a, const void* x, int64_t ld, int D, int bytes, hipStream_t s) {
  hipLaunchKernelGGL((k_micro_few<T, O>), dim3(((uint32_t)a.P + 63) / 64), dim3(256), bytes, s, a, (const T*)x, ld, D);
}

// The call's rows, from x (of type T) or, in the calls that bring them to codes first, a.x.
template <class O>
static void launch_micro_product(MicroArgs a, const void* x, int32_t type, int64_t ld, int D, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const int64_t few = a.N * ((a.blocks | 1) * 16 + a.sl);  // bytes of LDS
  if (a.N <= kFewRows && few <= 64 << 10) {
    if (type == WD_F32)
      launch_micro_few<F32, O>(a, x, ld, D, (int)few, s);
    else if (type == WD_F16)
      launch_micro_few<Half, O>(a, x, ld, D, (int)few, s);
    else
      launch_micro_few<Bf16, O>(a, x, ld, D, (int)few, s);
    return;
  }
  quantize(x, ld, a.N, D, type, codes, scales, s);
  // The largest tiles that fill the chip.  (128 x 128 and 64 x 64: 300 rows of 1024 to 100000 49.8 and 55.5 us, 2000
  // to 3001 16.5 and 16.6, 900 to 6000 15.2 and 15.3, 900 to 3001 12.6 and 10.9.  64 x 64 and 32 x 32: 300 rows to
  // 3001 8.1 and 8.4, 100 to 6000 7.7 and 7.5, 100 of 512 to 500 6.4 and 5.7.  32 x 64 for up to 32 rows: 32 rows
  // to 100000 15.0, in 64 x 64 16.6; 16 rows of 256 to 30000 5.5, in 32 x 32 6.0, to 6000 6.2 and 5.9.)
  const auto tiles = [&](int64_t m, int64_t n) { return ((a.N + m - 1) / m) * ((a.P + n - 1) / n); };
  a.stream = (uint64_t)a.N * a.P * sizeof(O) >= (256u << 20);
  if (a.N > 64 && tiles(128, 128) >= 384)
    launch_micro_tiles<O, 128, 128, 2, 2>(a, s);
  else if (a.N > 32 && tiles(64, 64) >= 192)
    launch_micro_tiles<O, 64, 64, 2, 2>(a, s);
  else if (a.N <= 32 && tiles(32, 64) >= 256)
    launch_micro_tiles<O, 32, 64, 1, 4>(a, s);
  else
    launch_micro_tiles<O, 32, 32, 2, 2>(a, s);
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
  type == WD_F32 ? launch_values<F32>(m, out, out_ld, (hipStream_t)stream) : launch_values<Bf16>(m, out, out_ld, (hipStream_t)stream);
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
  // (a launch has fewer than 2^32 threads: 2^24 workgroups of 256)
  const int64_t most = std::max<int64_t>(64, std::min<int64_t>(kMicroRows, (1ll << 23) / ((w->rows + 31) / 32) * 32));
  for (int64_t n0 = 0; n0 < N; n0 += most) {
    const int64_t n = std::min(most, N - n0);
    uint8_t *codes = (uint8_t*)ws, *scales = codes + align_up((uint64_t)n * micro_blocks(w->D) * 16, 256);
    const MicroArgs a{codes, scales, (const uint8_t*)w->codes, (const uint8_t*)w->scales, n, (int32_t)w->rows, (int32_t)micro_blocks(w->D),
                      (int32_t)micro_scales(w->D), bias, (char*)out + n0 * out_ld * oe, out_ld, false};
    const void* rows = (const char*)x + n0 * x_ld * xe;
    if (out_type == WD_F32)
      launch_micro_product<F32>(a, rows, type, x_ld, w->D, codes, scales, s);
    else if (out_type == WD_F16)
      launch_micro_product<Half>(a, rows, type, x_ld, w->D, codes, scales, s);
    else
      launch_micro_product<Bf16>(a, rows, type, x_ld, w->D, codes, scales, s);
  }
  return hip_check(hipGetLastError(), "micro_project");
}
