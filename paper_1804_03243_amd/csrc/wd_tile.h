// Products of matrices in tiles of matrix instructions: the operands' way through
// LDS, and the loop over the columns that two matrices share.
#pragma once

#include "wd_num.h"

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

// 16 bytes per lane from `base` (the same in every lane) + the lane's offset
// straight to LDS at `to` + 16 * lane (the same `to` in every lane).  The compiler
// does not see this load (its builtin makes every LDS read wait for all of them):
// the data is there after loads_left() and a barrier.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to) {
  const uint64_t p = (uint64_t)base;  // (into scalar registers, where the compiler would not hold it there)
  base = (const void*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 |
                       (uint32_t)__builtin_amdgcn_readfirstlane((int)p));
  to = (uint32_t)__builtin_amdgcn_readfirstlane((int)to);
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

constexpr int kStepK = 64;  // columns of a step: 128 bytes of a row

// Where chunk c (16 bytes) of tile row r lies in LDS: at c ^ swizzle, so that the
// 16 rows of an operand read fall on different banks.
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// The tile of a workgroup by its number.  Workgroups go round the eight XCDs, each with an
// L2 of its own: an XCD takes a run of tiles, in groups of kGroup (or group_rows) rows of tiles
// column by column, so that its workgroups share rows of x and of W.
constexpr uint32_t kGroup = 8;
__device__ __forceinline__ void tile_at(uint32_t number, uint32_t rows, uint32_t cols, uint32_t& row, uint32_t& col,
                                        uint32_t group_rows = kGroup) {
  const uint32_t all = rows * cols, xcd = number % 8, q = all / 8, r = all % 8;
  const uint32_t at = xcd * q + min(xcd, r) + number / 8;
  const uint32_t group = at / (group_rows * cols), first = group * group_rows, height = min(group_rows, rows - first);
  const uint32_t in = at - first * cols;
  col = in / height;
  row = first + in % height;
}
__device__ __forceinline__ void my_tile(uint32_t rows, uint32_t cols, uint32_t& row, uint32_t& col) { tile_at(blockIdx.x, rows, cols, row, col); }

// Zeros to load where a matrix has ended.
static __device__ const uint4 k_zeros[kStepK / 8] = {};

// One operand of a tile's product, from the tile's first row or column and the
// product's first shared column on.  By rows (KR = false) its memory has the shared
// columns side by side, `ld` bytes from row to row; by shared columns (KR = true) the
// tile's rows stand side by side, `ld` bytes from a shared column to the next.
// Either way 16-byte aligned, ld a multiple of 16, and `count` > 0 of the tile's rows
// exist: by rows, those past them repeat the last one; by shared columns, chunks of
// eight past them repeat the first chunk (a chunk that holds the last row is read as a
// whole: ld has room for it).
struct Operand {
  const void* p;
  int64_t ld;
  int count;
};

// Where rows 2c.. of a 16-row block of an operand by shared columns lie: chunk c of
// shared column k at c ^ turn(k).  A transposing read takes four columns k..k+3 for each
// quarter of the wavefront, eight columns apart: 16 pieces of 32 bytes, spread over the
// banks as far as the line (ROWS * 2 bytes) lets them.
template <int ROWS>
__device__ __forceinline__ int turn(int k) {
  if constexpr (ROWS >= 256) return ((k & 3) | ((k >> 3) & 3) << 2) * 2;
  if constexpr (ROWS == 128) return ((k & 3) | ((k >> 3) & 1) << 2) * 2;
  return ((k >> 1 & 1) | ((k >> 3) & 1) << 1) * 2;
}

// Transposing read of 16-bit values: within each 16 lanes, lane l gets value l % 4 of
// what the lanes 4 t + l / 4 address, t = 0..3.
__device__ __forceinline__ uint2 read_turned(uint32_t at) {
  typedef __attribute__((ext_vector_type(4))) short s16x4;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
}

// The wavefront's number, as a value that the compiler holds once for the wavefront.
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// The loads of one operand (of ROWS rows) by WAVES wavefronts, and a wavefront's reads of
// blocks of 16 rows from its first one, r0, on (a multiple of the rows that it has).
// Addresses are laid out so that a read costs an addition at most: blocks, halves and
// places are constants of the instruction or one bit of the address.
template <int ROWS, bool KR, int WAVES>
struct Side {
  static constexpr int kBytes = ROWS * 128;              // of a step
  static constexpr int kParts = kBytes / 1024 / WAVES;   // loads of a wavefront per step
  static constexpr int kChunks = KR ? ROWS / 8 : 8;      // chunks of a line in LDS
  static constexpr int kLines = 64 / kChunks;            // lines of a load
  static_assert(kBytes % (1024 * WAVES) == 0, "");
  Operand o;
  uint32_t from[kParts];
  uint32_t to;    // where the wavefront's first load goes
  uint32_t read;  // where the lane's first read is

  __device__ __forceinline__ void init(const Operand& op, int r0, uint32_t lds) {
    o = op;
    const int wave = wave_number(), lane = threadIdx.x & 63, quad = lane >> 4, l = lane & 15;
    to = lds + wave * 1024;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int line = (i * WAVES + wave) * kLines + lane / kChunks;
      if constexpr (KR) {
        const int c = (lane % kChunks) ^ turn<ROWS>(line);
        from[i] = (uint32_t)(line * o.ld + (c * 8 < o.count ? c * 16 : 0));
      } else {
        from[i] = (uint32_t)(min(line, o.count - 1) * o.ld + ((lane % kChunks) ^ swizzle(line)) * 16);
      }
    }
    if constexpr (KR) {
      const int k = quad * 8 + (l >> 2);
      read = lds + k * (ROWS * 2) + (((r0 / 8 | (l >> 1 & 1)) ^ turn<ROWS>(k)) << 4) + (l & 1) * 8;
    } else {
      read = lds + (r0 + l) * 128 + ((quad ^ swizzle(l)) << 4);
    }
  }
  // Starts the loads of shared columns k0.. of K (a multiple of eight by rows) to the step at `at`.
  __device__ __forceinline__ void stage(int k0, int K, int at) const {
    const char* base = (const char*)o.p + (KR ? (int64_t)k0 * o.ld : (int64_t)k0 * 2);
    if (k0 + kStepK <= K) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) load_to_lds(base, from[i], to + at + i * WAVES * 1024);
    } else {  // the last ones, zeros behind them
      const int lane = threadIdx.x & 63;
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        const int line = (i * WAVES + wave_number()) * kLines + lane / kChunks;
        const int k = k0 + (KR ? line : ((lane % kChunks) ^ swizzle(line)) * 8);
        if (k < K)
          load_to_lds(base, from[i], to + at + i * WAVES * 1024);
        else
          load_to_lds(k_zeros, 0, to + at + i * WAVES * 1024);
      }
    }
  }
  // The lane's eight columns of half h (0, 1) of the step at `at`, of row r0 + i * 16 + lane % 16.
  __device__ __forceinline__ uint4 rows(int at, int i, int h) const {
    if constexpr (KR) {
      const uint32_t p = (read ^ (i << 5)) + at + h * 32 * (ROWS * 2);
      const uint2 lo = read_turned(p), hi = read_turned(p + 4 * (ROWS * 2));
      return make_uint4(lo.x, lo.y, hi.x, hi.y);
    } else {
      typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
      const u32x4 v = *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)((read ^ (h << 6)) + at + i * 2048);
      return make_uint4(v.x, v.y, v.z, v.w);
    }
  }
};

// acc[i][j] += the products of x's rows (BM of the tile, TM blocks of 16 a wavefront)
// with w's (BN, TN blocks) over K shared columns.  w is the matrix instruction's first
// operand, so that a lane holds four consecutive rows of w (outputs, quad * 4 ..) of one
// row of x (lane % 16).  Two steps of kStepK columns are in LDS.  A step is two halves:
// while one is multiplied, the next half's operands are read into registers; between
// the halves of a step every wavefront has read all of it, and the step after the next
// starts into its place.  (Three or four steps in LDS in the smallest tiles: no faster,
// and up to 17% slower.)  What the caller has written to other LDS before is there behind it
// for every wavefront; kBytes of `lds` are free again after a barrier.
// EXACT: the sums of four steps are formed by themselves and added up with what each
// addition rounds off, so that a sum is off by the roundings within four steps and one more.
template <class T, int BM, int BN, int WM, int WN, bool XKR, bool WKR, bool EXACT = false>
struct Tile {
  static constexpr int kWaves_ = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr int kStep = (BM + BN) * 128, kBytes = 2 * kStep;
  using X = Side<BM, XKR, kWaves_>;
  using W = Side<BN, WKR, kWaves_>;

  static __device__ __forceinline__ void multiply(const Operand& xo, const Operand& wo, int K, char* lds, f32x4 (&acc)[TM][TN]) {
    const int wave = wave_number(), wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    X x;
    W w;
    x.init(xo, wm, lds0);
    w.init(wo, wn, lds0 + X::kBytes);
    const auto stage = [&](int k0, int at) {
      x.stage(k0, K, at);
      w.stage(k0, K, at);
    };
    struct Operands {
      uint4 w[TN], x[TM];
    } even, odd;
    const auto read = [&](int at, int half, Operands& o) {
#pragma unroll
      for (int j = 0; j < TN; ++j) o.w[j] = w.rows(at, j, half);
#pragma unroll
      for (int i = 0; i < TM; ++i) o.x[i] = x.rows(at, i, half);
    };
    f32x4 part[EXACT ? TM : 1][EXACT ? TN : 1] = {}, off[EXACT ? TM : 1][EXACT ? TN : 1] = {};
    const auto products = [&](const Operands& o) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if constexpr (EXACT)
            part[i][j] = mfma16(o.w[j], o.x[i], part[i][j], T{});
          else
            acc[i][j] = mfma16(o.w[j], o.x[i], acc[i][j], T{});
      // an operand read between every few products
      constexpr int kReads = TM * (XKR ? 2 : 1) + TN * (WKR ? 2 : 1), kEach = TM * TN / kReads > 0 ? TM * TN / kReads : 1;
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
      }
    };
    const auto add = [&]() {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = acc[i][j][e], b = part[i][j][e], s = a + b, v = s - a, r = (a - (s - v)) + (b - v);
            acc[i][j][e] = s;
            off[i][j][e] += fabsf(r) < INFINITY ? r : 0.0f;  // (sums that are not finite stay as they are)
            part[i][j][e] = 0.0f;
          }
    };
    int now = 0, next = kStep;
    stage(0, now);
    if (kStepK < K) {
      stage(kStepK, next);
      2 * kStepK <= K ? loads_left<X::kParts + W::kParts>() : loads_left<0>();
    } else {
      loads_left<0>();
    }
    __syncthreads();
    read(now, 0, even);
    // (One copy of the products and no branch around them: with more the compiler
    // holds the accumulators twice.  The last step's reads of a next one are of no use.)
    for (int k0 = 0; k0 < K; k0 += kStepK) {
      read(now, 1, odd);
      products(even);
      loads_left<0>();
      __syncthreads();  // this step has been read, the next one is there
      if (k0 + 2 * kStepK < K) stage(k0 + 2 * kStepK, now);
      read(next, 0, even);
      products(odd);
      if constexpr (EXACT)
        if (k0 / kStepK % 4 == 3 || k0 + kStepK >= K) add();
      now = next;
      next = kStep - next;
    }
    if constexpr (EXACT) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] += off[i][j];
    }
  }
};

// A tile's values to memory, a block of 16 rows at a time through LDS (`mine`, the
// wavefront's own), so that a store instruction writes whole lines of a row.  value(i, j, e)
// is the lane's value of row i * 16 + lane % 16, column j * 16 + lane / 16 * 4 + e.
// `stream`: past the caches, for outputs larger than they are.
template <class O, int TM, int TN, class Value>
__device__ __forceinline__ void store_tile(O* out, int64_t ld, int64_t rows, int64_t cols, char* mine, Value value, bool stream = false) {
  constexpr int kCols = TN * 16, kEach = 16 / sizeof(O);
  constexpr int kLine = kCols + kEach;  // a row in LDS, padded against bank conflicts
  constexpr int kLanes = kCols / kEach, kRows = 64 / kLanes;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  O* lines = (O*)mine;
  const int c = (lane % kLanes) * kEach, r0 = lane / kLanes, left = (int)min<int64_t>(cols - c, kEach);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      struct alignas(4 * sizeof(O)) Four {
        O v[4];
      } v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v.v[e] = O::of(value(i, j, e));
      *(Four*)(lines + col * kLine + j * 16 + quad * 4) = v;
    }
#pragma unroll
    for (int q = 0; q < 16; q += kRows) {
      if (kRows > 16 && r0 >= 16) continue;  // (16 columns of 16 bits: half the lanes)
      const uint4 v = *(const uint4*)(lines + (q + r0) * kLine + c);
      const int64_t n = i * 16 + q + r0;
      if (n < rows) {
        if (stream && left >= kEach)
          __builtin_nontemporal_store(__builtin_bit_cast(f32x4, v), (f32x4_any*)(out + n * ld + c));
        else
          store_out(out + n * ld + c, __builtin_bit_cast(Few<O, kEach>, v), left);
      }
    }
  }
}
// Bytes of store_tile's LDS for each wavefront.
template <class O, int TN>
constexpr int kStoreBytes = 16 * (TN * 16 + 16 / (int)sizeof(O)) * (int)sizeof(O);

}  // namespace wd
