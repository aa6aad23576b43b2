// Logits to log-likelihoods: penalties for labels a request has had, its
// biases, its row's label mask, log-softmax, log priors and the acoustic scale.
//
// A workgroup holds a row, or a slice of one, in registers.  Its penalties need the
// count of each label in the request's history, its biases the last entry of
// the label: both lists are scattered into one table of the slice's labels in LDS, the
// last entry as the maximum of the entries' positions in the upper 16 bits, then the
// count by additions in the lower ones (integer atomics: the order of the entries
// does not matter; longer lists take the table in turn).  Then m = max z and s = sum
// of exp(z - m) over the workgroup, in 32 bits, and y = (z - m) - log s.  Bound by
// memory where rows are many (67 thousand rows of 6000 labels of 32 bits: 590 us, 5.5
// TB/s, a little more than a copy reaches), by the chain of reads request, offsets, list
// where they are few.
#include <algorithm>
#include <cmath>

#include "wd_host.h"
#include "wd_num.h"

namespace wd {

struct ScoreArgs {
  wd_loglikes_args a;
  float2* part;     // [N][slices] maximum and sum of each slice of a row
  uint32_t slices;  // slices of a row
  bool stream;      // outputs past the caches
};

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// A finite number to subtract from logits of maximum m before their exponentials
// are taken: with nothing above -inf, exp(z - 0) = 0 and a NaN stays one.
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.0f : m; }

struct RowSpan {
  int64_t b, e;
};
__device__ __forceinline__ RowSpan span_of(const int64_t* off, int q, int64_t n) {
  return {max(off[q], (int64_t)0), min(off[q + 1], n)};
}

// Four consecutive elements of a row of n, those past its end as `fill`.
template <class T>
__device__ __forceinline__ Few<T, 4> load4(const T* p, int n, T fill) {
  if (n >= 4) return *(const Few<T, 4>*)p;
  Few<T, 4> v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v.v[i] = i < n ? p[i] : fill;
  return v;
}

// What a workgroup does with its slice of a row.
enum ScorePhase {
  kWhole,  // the slice is the row: normalise and write
  kStats,  // its maximum and sum, to `part`
  kWrite   // write, with the sums of all slices from `part`
};

// A workgroup per slice of THREADS * EACH labels, a thread's labels in registers:
// (j * THREADS + thread) * 4 + i of the slice is z[j * 4 + i].
template <class T, int THREADS, int EACH, ScorePhase PHASE, bool LISTS>
__global__ void __launch_bounds__(THREADS) k_loglikes(ScoreArgs args) {
  constexpr int kSlice = THREADS * EACH, kVecs = EACH / 4, kWavesHere = THREADS / 64;
  const wd_loglikes_args& a = args.a;
  extern __shared__ uint32_t table[];  // [kSlice], where there are histories or biases
  __shared__ float red[2][kWavesHere];
  const int64_t n = PHASE == kWhole ? blockIdx.x : blockIdx.x / args.slices;
  const int c0 = PHASE == kWhole ? 0 : (int)(blockIdx.x % args.slices) * kSlice;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t to = n;
  if (a.out_row) {
    to = a.out_row[n];
    if (to < 0 || to >= a.out_rows) return;
  }
  int q = -1;
  if (a.n_requests > 0) {
    const int64_t r = a.request ? (int64_t)a.request[n] : n;
    q = r >= 0 && r < a.n_requests ? (int)r : -1;
  }
  RowSpan hist{0, 0}, bias{0, 0};
  if (LISTS && q >= 0 && a.hist_off) hist = span_of(a.hist_off, q, a.n_hist);
  if (LISTS && q >= 0 && a.bias_off) bias = span_of(a.bias_off, q, a.n_bias);
  const int V = a.V, at = c0 + (int)threadIdx.x * 4;
  constexpr int kStep = THREADS * 4;
  const T* row = (const T*)a.logits + n * a.ld;
  Few<T, 4> raw[kVecs];
#pragma unroll
  for (int j = 0; j < kVecs; ++j) raw[j] = load4(row + at + j * kStep, V - at - j * kStep, T::of(-INFINITY));

  uint32_t keep[kVecs];  // bits of the mask
  const uint32_t* mask = nullptr;
  if (a.mask) {
    const int64_t r = a.mask_of ? (int64_t)a.mask_of[n] : n;
    if (r >= 0 && r < a.n_masks) mask = a.mask + r * a.mask_ld;
  }
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int v = at + j * kStep;
    keep[j] = mask && v < V ? mask[v >> 5] >> (v & 31) : 15u;
  }

  float z[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) z[j] = raw[j / 4].v[j & 3].f();
  const bool has_hist = hist.b < hist.e, has_bias = bias.b < bias.e;  // (the same for the whole workgroup)
  if (LISTS && (has_hist || has_bias)) {
    // (a product with the rounded reciprocal is off by up to 1.5 units of the last place,
    // a quotient by half a one: one instruction a label for about ten)
    const float rho = has_hist && a.repetition ? a.repetition[q] : 1.0f, inv_rho = 1.0f / rho;
    const float pres = has_hist && a.presence ? a.presence[q] : 0.0f, freq = has_hist && a.frequency ? a.frequency[q] : 0.0f;
    const auto clear = [&]() {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) ((uint4*)table)[j * THREADS + threadIdx.x] = make_uint4(0, 0, 0, 0);
      __syncthreads();
    };
    const auto inside = [&](int l) { return l < V && (uint32_t)(l - c0) < (uint32_t)kSlice; };
    const auto place = [&](int shift) {
#pragma unroll 4
      for (int64_t i = bias.b + threadIdx.x; i < bias.e; i += THREADS) {
        const int l = a.bias_id[i];
        if (inside(l)) atomicMax(&table[l - c0], ((uint32_t)(i - bias.b) + 1u) << shift);
      }
      __syncthreads();
    };
    const auto count = [&]() {
#pragma unroll 4
      for (int64_t i = hist.b + threadIdx.x; i < hist.e; i += THREADS) {
        const int l = a.hist[i];
        if (inside(l)) atomicAdd(&table[l - c0], 1u);
      }
      __syncthreads();
    };
    // of each label: how often it stands in the history (e & counts), and which bias it has (e >> places)
    const auto apply = [&](uint32_t counts, int places) {
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        const uint4 e4 = ((const uint4*)table)[j * THREADS + threadIdx.x];
        if (!(e4.x | e4.y | e4.z | e4.w)) continue;
        const uint32_t e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float& x = z[j * 4 + i];
          const uint32_t c = e[i] & counts, p = (uint32_t)((uint64_t)e[i] >> places);
          if (c) x = x * (x > 0.0f ? inv_rho : rho) - (pres + freq * (float)c);
          if (p) x += a.bias_val[bias.b + (p - 1)];
        }
      }
    };
    // both lists at once, or one after the other where one is too long for 16 bits
    const bool both = hist.e - hist.b < 65536 && bias.e - bias.b < 65536;
#pragma unroll 1
    for (int pass = 0; pass < (both ? 1 : 2); ++pass) {
      const bool counts = has_hist && pass == 0, places = has_bias && (both || pass == 1);
      if (pass) __syncthreads();
      clear();
      if (places) place(both ? 16 : 0);
      if (counts) count();
      apply(!counts ? 0u : both ? 0xffffu : 0xffffffffu, !places ? 32 : both ? 16 : 0);
    }
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j)
    if (!(keep[j / 4] >> (j & 3) & 1u)) z[j] = -INFINITY;

  float m = 0.0f, lse = 0.0f;
  if (PHASE != kWrite && a.normalize) {
    m = -INFINITY;
#pragma unroll
    for (int j = 0; j < EACH; ++j) m = fmaxf(m, z[j]);
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) red[0][wave] = m;
    __syncthreads();
    m = red[0][0];
#pragma unroll
    for (int w = 1; w < kWavesHere; ++w) m = fmaxf(m, red[0][w]);
    const float top = m;
    m = shift_of(m);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < EACH; ++j) s += exp_of(z[j] - m);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) red[1][wave] = s;
    __syncthreads();
    s = red[1][0];
#pragma unroll
    for (int w = 1; w < kWavesHere; ++w) s += red[1][w];
    if (PHASE == kStats) {
      if (threadIdx.x == 0) args.part[blockIdx.x] = make_float2(top, s);
      return;
    }
    lse = logf(s);
  }
  if (PHASE == kWrite && a.normalize) {
    const float2* p = args.part + n * args.slices;
    m = -INFINITY;
    for (uint32_t i = lane; i < args.slices; i += 64) m = fmaxf(m, p[i].x);
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    m = shift_of(m);
    float s = 0.0f;
    for (uint32_t i = lane; i < args.slices; i += 64) s += p[i].y == 0.0f ? 0.0f : p[i].y * exp_of(shift_of(p[i].x) - m);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    lse = logf(s);
  }
  float* out = a.out + to * a.out_ld;
#pragma unroll
  for (int j = 0; j < kVecs; ++j) {
    const int v = at + j * kStep;
    if (v >= V) break;
    Few<F32, 4> prior{};
    if (a.log_prior) prior = load4((const F32*)a.log_prior + v, V - v, F32{0.0f});
    f32x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = z[j * 4 + i];
      y[i] = x == -INFINITY ? x : a.scale * (((x - m) - lse) - prior.v[i].u);
    }
    if (V - v >= 4) {
      if (args.stream)
        __builtin_nontemporal_store(y, (f32x4_any*)(out + v));
      else
        *(f32x4_any*)(out + v) = y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (v + i < V) out[v + i] = y[i];
    }
  }
}

// Rows of up to kWholeLabels labels are one slice: they are read once and their
// lists are scattered once (400 rows of 30000 labels of 16 bits with histories and
// biases, whole call: 33 us, in slices 48; 8 rows 13.6 and 16.7).  Longer ones go
// in slices, twice (400 rows of 100000 labels: 109 us in slices of 8192 labels, 153
// of 16384, 173 of 32768: more workgroups hide each other's waits for the lists).
// A row's workgroup is the smallest that holds it (4000 rows of 16 bits with lists of
// 500: 2048 labels 24 us by 256 threads of 8 and 27 of 16; 4096 35 by 256 of 16, 51 of 32;
// 8192 72 by 256 of 32 and 98 by 1024 of 8 - 63 by 512 of 16 -; 16384 190 by 1024 of 16,
// 231 of 32).  One row or 64 take the same time either way, to 1 us.
constexpr int kWholeLabels = 32768;
constexpr int kSliceThreads = 512, kSliceEach = 16, kSliceLabels = kSliceThreads * kSliceEach;

// The arguments without their first n rows.
inline ScoreArgs rows_from(ScoreArgs args, int64_t n) {
  wd_loglikes_args& a = args.a;
  a.N -= n;
  a.logits = (const char*)a.logits + n * a.ld * (a.type == WD_F32 ? 4 : 2);
  args.part = args.part ? args.part + n * args.slices : nullptr;
  if (a.out_row)
    a.out_row += n;
  else
    a.out += n * a.out_ld;
  if (a.request) {
    a.request += n;
  } else {  // (row n is request n)
    a.n_requests = (int32_t)std::max<int64_t>(0, a.n_requests - n);
    if (a.hist_off) a.hist_off += n;
    if (a.bias_off) a.bias_off += n;
    if (a.repetition) a.repetition += n;
    if (a.presence) a.presence += n;
    if (a.frequency) a.frequency += n;
  }
  if (a.mask_of) {
    a.mask_of += n;
  } else if (a.mask) {
    a.n_masks = std::max<int64_t>(0, a.n_masks - n);
    a.mask += n * a.mask_ld;
  }
  return args;
}

// (A launch has fewer than 2^32 threads: more rows than that take several.)
template <class T, int THREADS, int EACH, ScorePhase PHASE>
void launch_slices(const ScoreArgs& all, hipStream_t s) {
  const int64_t most = (((int64_t)1 << 32) / THREADS - 1) / all.slices;
  for (int64_t n0 = 0; n0 < all.a.N; n0 += most) {
    const ScoreArgs args = n0 ? rows_from(all, n0) : all;
    const dim3 grid((uint32_t)(std::min(most, args.a.N) * args.slices)), block(THREADS);
    if (!args.a.hist_off && !args.a.bias_off) {
      hipLaunchKernelGGL((k_loglikes<T, THREADS, EACH, PHASE, false>), grid, block, 0, s, args);
      continue;
    }
    auto* k = k_loglikes<T, THREADS, EACH, PHASE, true>;
    static std::atomic<uint64_t> done{0};
    allow_lds((const void*)k, THREADS * EACH * 4, done);
    hipLaunchKernelGGL(k, grid, block, THREADS * EACH * 4, s, args);
  }
}

template <class T>
void launch_loglikes(const wd_loglikes_args* a, void* ws, hipStream_t s) {
  ScoreArgs args{*a, (float2*)ws, 1, (uint64_t)a->N * a->V * 4 >= (256u << 20)};
  if (a->V <= 2048)
    launch_slices<T, 256, 8, kWhole>(args, s);
  else if (a->V <= 4096)
    launch_slices<T, 256, 16, kWhole>(args, s);
  else if (a->V <= 8192)
    launch_slices<T, 256, 32, kWhole>(args, s);
  else if (a->V <= 16384)
    launch_slices<T, 1024, 16, kWhole>(args, s);
  else if (a->V <= kWholeLabels)
    launch_slices<T, 1024, 32, kWhole>(args, s);
  else {
    args.slices = (uint32_t)((a->V + kSliceLabels - 1) / kSliceLabels);
    if (a->normalize) launch_slices<T, kSliceThreads, kSliceEach, kStats>(args, s);
    launch_slices<T, kSliceThreads, kSliceEach, kWrite>(args, s);
  }
}

}  // namespace wd

using namespace wd;

static wd_status check_loglikes(const wd_loglikes_args* a) {
  if (!a) return fail(WD_EINVAL, "loglikes: null arguments");
  if (a->V < 1 || a->V >= (1 << 24)) return fail(WD_EINVAL, "loglikes: V out of range");
  if (a->N < 0 || a->N > INT32_MAX / (a->V / kSliceLabels + 1)) return fail(WD_EINVAL, "loglikes: N out of range");
  if (a->type != WD_F32 && a->type != WD_F16 && a->type != WD_BF16) return fail(WD_EINVAL, "loglikes: unknown type");
  if (a->ld < a->V || a->out_ld < a->V) return fail(WD_EINVAL, "loglikes: row stride below V");
  if (!(a->scale > 0.0f) || std::isinf(a->scale)) return fail(WD_EINVAL, "loglikes: scale must be finite and > 0");
  if (a->n_requests < 0 || a->n_hist < 0 || a->n_bias < 0 || a->n_masks < 0 || a->out_rows < 0)
    return fail(WD_EINVAL, "loglikes: negative count");
  if (a->n_bias >= (int64_t)0xffffffffu) return fail(WD_EINVAL, "loglikes: too many biases");
  if (a->N == 0) return WD_OK;
  if (!a->logits || !a->out) return fail(WD_EINVAL, "loglikes: null logits or output");
  if ((a->hist_off || a->bias_off) && a->n_requests == 0)
    return fail(WD_EINVAL, "loglikes: histories or biases without requests");
  if (a->hist_off && a->n_hist && !a->hist) return fail(WD_EINVAL, "loglikes: null history");
  if (a->bias_off && a->n_bias && (!a->bias_id || !a->bias_val)) return fail(WD_EINVAL, "loglikes: null biases");
  if (a->mask && a->mask_ld < ((int64_t)a->V + 31) / 32) return fail(WD_EINVAL, "loglikes: mask_ld below ceil(V / 32)");
  if (!a->out_row && a->out_rows < a->N) return fail(WD_EINVAL, "loglikes: fewer output rows than rows");
  const uintptr_t e = a->type == WD_F32 ? 3 : 1;
  if ((uintptr_t)a->logits & e || (uintptr_t)a->out & 3) return fail(WD_EINVAL, "loglikes: misaligned logits or output");
  const void* w4[] = {a->log_prior, a->request, a->hist, a->repetition, a->presence, a->frequency,
                      a->bias_id, a->bias_val, a->mask, a->mask_of, a->out_row};
  for (const void* p : w4)
    if ((uintptr_t)p & 3) return fail(WD_EINVAL, "loglikes: misaligned array");
  if ((uintptr_t)a->hist_off & 7 || (uintptr_t)a->bias_off & 7) return fail(WD_EINVAL, "loglikes: misaligned offsets");
  return WD_OK;
}

// Workspace: the slices' maxima and sums.
static size_t parts_bytes(const wd_loglikes_args* a) {
  if (a->V <= kWholeLabels || !a->normalize) return 0;
  return align_up((uint64_t)a->N * ((a->V + kSliceLabels - 1) / kSliceLabels) * sizeof(float2), 256);
}

extern "C" wd_status wd_loglikes_workspace_bytes(const wd_loglikes_args* a, size_t* bytes) {
  if (!bytes) return fail(WD_EINVAL, "loglikes_workspace_bytes: null output");
  wd_status st = check_loglikes(a);
  if (st != WD_OK) return st;
  *bytes = parts_bytes(a);
  return WD_OK;
}

extern "C" wd_status wd_loglikes(const wd_loglikes_args* a, void* ws, size_t ws_bytes, void* stream) {
  wd_status st = check_loglikes(a);
  if (st != WD_OK || a->N == 0) return st;
  const size_t need = parts_bytes(a);
  if (need && (!ws || ws_bytes < need || (uintptr_t)ws & 255))
    return fail(WD_EINVAL, "loglikes: workspace missing, too small or not 256-byte aligned");
  hipStream_t s = (hipStream_t)stream;
  if (a->type == WD_F32)
    launch_loglikes<F32>(a, ws, s);
  else if (a->type == WD_F16)
    launch_loglikes<Half>(a, ws, s);
  else
    launch_loglikes<Bf16>(a, ws, s);
  return hip_check(hipGetLastError(), "loglikes");
}
