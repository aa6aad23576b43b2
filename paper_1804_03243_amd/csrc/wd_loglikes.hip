// Logits to log-likelihoods: penalties for labels a request has had, its
// biases, its row's label mask, log-softmax, log priors and the acoustic scale.
//
// A row is swept in chunks of labels.  A chunk's penalties need the count of
// each label in the request's history: the history is scattered into a
// table of the chunk's labels in LDS (integer atomics: the order of the entries
// does not matter), and the last bias entry of a label is the maximum of the
// entries' positions in the same table.  The log of the sum of exponentials is
// kept as a running maximum m and a running sum s of exp(z - m) per thread, in
// 32 bits; rows of more than one chunk are swept twice.
#include <algorithm>
#include <cmath>

#include "wd_host.h"
#include "wd_num.h"

namespace wd {

constexpr int kScoreThreads = 256;
constexpr int kScoreEach = 32;                       // labels of a chunk per thread
constexpr int kScoreChunk = kScoreThreads * kScoreEach;

struct ScoreArgs {
  wd_loglikes_args a;
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

struct RowSpan {
  int64_t b, e;
};

__device__ __forceinline__ RowSpan span_of(const int64_t* off, int q, int64_t n) {
  return {max(off[q], (int64_t)0), min(off[q + 1], n)};
}

// The adjusted logits of the chunk's labels c0 + (j * threads + thread) * 4 + i
// in z[j * 4 + i]; -inf past the row.
template <class T>
__device__ __forceinline__ void score_chunk(const wd_loglikes_args& a, const T* row, int q, const uint32_t* mask, int c0,
                                            uint32_t* table, float* z) {
  const int V = a.V;
#pragma unroll
  for (int j = 0; j < kScoreEach / 4; ++j) {
    const int v = c0 + (j * kScoreThreads + (int)threadIdx.x) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) z[j * 4 + i] = v + i < V ? row[v + i].f() : -INFINITY;
  }
  if (q >= 0 && a.hist_off) {
    const RowSpan h = span_of(a.hist_off, q, a.n_hist);
    if (h.b < h.e) {  // (the same for the whole workgroup)
      for (int i = threadIdx.x; i < kScoreChunk; i += kScoreThreads) table[i] = 0;
      __syncthreads();
      for (int64_t i = h.b + threadIdx.x; i < h.e; i += kScoreThreads) {
        const int l = a.hist[i];
        if (l >= c0 && l < V && l - c0 < kScoreChunk) atomicAdd(&table[l - c0], 1u);
      }
      __syncthreads();
      const float rho = a.repetition ? a.repetition[q] : 1.0f;
      const float pres = a.presence ? a.presence[q] : 0.0f, freq = a.frequency ? a.frequency[q] : 0.0f;
#pragma unroll
      for (int j = 0; j < kScoreEach; ++j) {
        const uint32_t c = table[((j >> 2) * kScoreThreads + (int)threadIdx.x) * 4 + (j & 3)];
        if (c) z[j] = (z[j] > 0.0f ? z[j] / rho : z[j] * rho) - (pres + freq * (float)c);
      }
      __syncthreads();
    }
  }
  if (q >= 0 && a.bias_off) {
    const RowSpan h = span_of(a.bias_off, q, a.n_bias);
    if (h.b < h.e) {
      for (int i = threadIdx.x; i < kScoreChunk; i += kScoreThreads) table[i] = 0;
      __syncthreads();
      for (int64_t i = h.b + threadIdx.x; i < h.e; i += kScoreThreads) {
        const int l = a.bias_id[i];
        if (l >= c0 && l < V && l - c0 < kScoreChunk) atomicMax(&table[l - c0], (uint32_t)(i - h.b) + 1u);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kScoreEach; ++j) {
        const uint32_t c = table[((j >> 2) * kScoreThreads + (int)threadIdx.x) * 4 + (j & 3)];
        if (c) z[j] += a.bias_val[h.b + (c - 1)];
      }
      __syncthreads();
    }
  }
  if (mask) {
#pragma unroll
    for (int j = 0; j < kScoreEach / 4; ++j) {
      const int v = c0 + (j * kScoreThreads + (int)threadIdx.x) * 4;
      const uint32_t w = v < V ? mask[v >> 5] >> (v & 31) : 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!((w >> i) & 1u)) z[j * 4 + i] = -INFINITY;
    }
  }
}

template <class T>
__global__ void __launch_bounds__(kScoreThreads) k_loglikes(ScoreArgs args) {
  const wd_loglikes_args& a = args.a;
  __shared__ uint32_t table[kScoreChunk];
  __shared__ float red[2 * kScoreThreads];
  for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
    int64_t to = n;
    if (a.out_row) {
      to = a.out_row[n];
      if (to < 0 || to >= a.out_rows) continue;
    }
    const T* row = (const T*)a.logits + n * a.ld;
    float* out = a.out + to * a.out_ld;
    int q = -1;
    if (a.n_requests > 0) {
      const int64_t r = a.request ? (int64_t)a.request[n] : n;
      q = r >= 0 && r < a.n_requests ? (int)r : -1;
    }
    const uint32_t* mask = nullptr;
    if (a.mask) {
      const int64_t r = a.mask_of ? (int64_t)a.mask_of[n] : n;
      if (r >= 0 && r < a.n_masks) mask = a.mask + r * a.mask_ld;
    }
    float z[kScoreEach];
    float m = -INFINITY, s = 0.0f, lse = 0.0f;
    if (a.normalize) {
      for (int c0 = 0; c0 < a.V; c0 += kScoreChunk) {
        score_chunk(a, row, q, mask, c0, table, z);
        float cm = m;
#pragma unroll
        for (int j = 0; j < kScoreEach; ++j) cm = fmaxf(cm, z[j]);
        const float base = cm == -INFINITY ? 0.0f : cm;  // nothing above -inf: exp(z - 0) = 0, a NaN stays one
        s = s == 0.0f ? 0.0f : s * exp_of(m - base);
#pragma unroll
        for (int j = 0; j < kScoreEach; ++j) s += exp_of(z[j] - base);
        m = cm;
      }
      red[threadIdx.x] = m;
      red[kScoreThreads + threadIdx.x] = s;
      __syncthreads();
      for (int w = kScoreThreads / 2; w > 0; w >>= 1) {
        if ((int)threadIdx.x < w) {
          const float m0 = red[threadIdx.x], m1 = red[threadIdx.x + w];
          const float mm = fmaxf(m0, m1), base = mm == -INFINITY ? 0.0f : mm;
          const float s0 = red[kScoreThreads + threadIdx.x], s1 = red[kScoreThreads + threadIdx.x + w];
          red[threadIdx.x] = mm;
          red[kScoreThreads + threadIdx.x] = (s0 == 0.0f ? 0.0f : s0 * exp_of(m0 - base)) + (s1 == 0.0f ? 0.0f : s1 * exp_of(m1 - base));
        }
        __syncthreads();
      }
      m = red[0] == -INFINITY ? 0.0f : red[0];
      lse = logf(red[kScoreThreads]);
      __syncthreads();
    } else {
      m = 0.0f;
    }
    for (int c0 = 0; c0 < a.V; c0 += kScoreChunk) {
      if (!a.normalize || a.V > kScoreChunk) score_chunk(a, row, q, mask, c0, table, z);
#pragma unroll
      for (int j = 0; j < kScoreEach; ++j) {
        const int v = c0 + ((j >> 2) * kScoreThreads + (int)threadIdx.x) * 4 + (j & 3);
        if (v < a.V) {
          const float y = (z[j] - m) - lse - (a.log_prior ? a.log_prior[v] : 0.0f);
          out[v] = z[j] == -INFINITY ? z[j] : a.scale * y;
        }
      }
    }
  }
}

}  // namespace wd

using namespace wd;

static wd_status check_loglikes(const wd_loglikes_args* a) {
  if (!a) return fail(WD_EINVAL, "loglikes: null arguments");
  if (a->N < 0) return fail(WD_EINVAL, "loglikes: negative N");
  if (a->V < 1 || a->V >= (1 << 24)) return fail(WD_EINVAL, "loglikes: V out of range");
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

extern "C" wd_status wd_loglikes_workspace_bytes(const wd_loglikes_args* a, size_t* bytes) {
  if (!bytes) return fail(WD_EINVAL, "loglikes_workspace_bytes: null output");
  wd_status st = check_loglikes(a);
  if (st != WD_OK) return st;
  *bytes = 0;
  return WD_OK;
}

extern "C" wd_status wd_loglikes(const wd_loglikes_args* a, void* ws, size_t ws_bytes, void* stream) {
  wd_status st = check_loglikes(a);
  if (st != WD_OK || a->N == 0) return st;
  (void)ws;
  (void)ws_bytes;
  const ScoreArgs args{*a};
  const dim3 grid((uint32_t)std::min<int64_t>(a->N, 1 << 20)), block(kScoreThreads);
  hipStream_t s = (hipStream_t)stream;
  if (a->type == WD_F32)
    hipLaunchKernelGGL(k_loglikes<F32>, grid, block, 0, s, args);
  else if (a->type == WD_F16)
    hipLaunchKernelGGL(k_loglikes<Half>, grid, block, 0, s, args);
  else
    hipLaunchKernelGGL(k_loglikes<Bf16>, grid, block, 0, s, args);
  return hip_check(hipGetLastError(), "loglikes");
}
