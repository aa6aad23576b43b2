// Label masks from the decoding graph: for every row, the input labels that
// leave a set of states, as bits.
//
//   mask[n] = OR over s in states(n), over arcs a of s with ilabel k >= 1, of bit k - 1
//
// The caller's arcs of a state are a run of the label array (by caller arc
// id), which starts at the number of emitting plus epsilon arcs before it, so
// an arc costs a 4-byte read; one or two arcs (most states of a decoding graph)
// stand in the state's offset record itself.  A row's bits are gathered in LDS.
// Bound by the scattered reads, which miss the L2 (16000 sets of 100 states among
// 500000: 34 us; 10 without them).  A lane reads up to eight labels of its own
// state with two loads; what states with more arcs have left is dealt out over the
// lanes, four reads of a lane at a time (300 sets of 20000 states of 3 arcs on average
// and up to hundreds: 93 us; one at a time 107).
#include <algorithm>

#include "wd_host.h"
#include "wd_num.h"

namespace wd {

struct LabelArgs {
  const uint4* off;
  const int32_t* ilabel;
  uint32_t S, words, parts;
  int64_t A, N, n_states, ld;
  const int64_t* row;
  const int32_t* states;
  uint32_t* mask;
};

// Four labels from `at` on, those past the label array's end as epsilon.
__device__ __forceinline__ Few<int32_t, 4> labels_at(const LabelArgs& a, uint32_t at) {
  if (a.A - at >= 4) return *(const Few<int32_t, 4>*)(a.ilabel + at);
  Few<int32_t, 4> v{};
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (at + i < a.A) v.v[i] = a.ilabel[at + i];
  return v;
}

// The bits of up to 64 states, one per lane; `deal` is LDS of the wavefront's own.
constexpr uint32_t kOwnArcs = 8;  // arcs that a lane reads itself
__device__ __forceinline__ void add_labels(const LabelArgs& a, uint32_t s, uint32_t* bits, uint2* deal) {
  const auto set = [&](int32_t label) {
    const uint32_t l = (uint32_t)label - 1u;  // (epsilon: out of range)
    if (l < a.words * 32u) atomicOr(&bits[l >> 5], 1u << (l & 31));
  };
  uint32_t first = 0, count = 0;
  if (s < a.S) {
    const uint4 o = a.off[s];
    first = o.x + o.y;
    const uint32_t kind = o.w >> 30;  // (state_arcs)
    if (kind) {
      set(kind == 1 ? o.w & 0xffffffu : o.w & 0x7fffu);
      if (kind == 2) set(o.w >> 15 & 0x7fffu);
    } else {
      count = o.w;
      if (count == kManyArcs) count = a.off[s + 1].x + a.off[s + 1].y - first;
    }
  }
  Few<int32_t, 4> v[2] = {};
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (count > 4u * k) v[k] = labels_at(a, first + 4 * k);
#pragma unroll
  for (int i = 0; i < (int)kOwnArcs; ++i)
    if ((uint32_t)i < count) set(v[i / 4].v[i & 3]);
  uint32_t more = count > kOwnArcs ? count - kOwnArcs : 0, at = first + kOwnArcs;
  while (__any(more != 0)) {
    // item i of the rest belongs to the last lane whose items start at or before i
    const uint32_t now = min(more, 1u << 25);  // (64 lanes' items stay below 2^32)
    const uint32_t end = wave_incl_scan(now), total = lane63(end), start = end - now;
    deal[lane_id()] = make_uint2(start, at - start);
    __builtin_amdgcn_wave_barrier();
    const auto arc = [&](uint32_t i) {
      uint32_t owner = 0;
#pragma unroll
      for (uint32_t step = 32; step > 0; step >>= 1)
        if (deal[owner + step].x <= i) owner += step;
      return i + deal[owner].y;
    };
    uint32_t i = lane_id();
    for (; (i | 63) + 192 < total; i += 256) {  // (four reads under way)
      int32_t l[4];
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) l[k] = a.ilabel[arc(i + 64 * k)];
#pragma unroll
      for (uint32_t k = 0; k < 4; ++k) set(l[k]);
    }
    for (; i < total; i += 64) set(a.ilabel[arc(i)]);
    __builtin_amdgcn_wave_barrier();
    more -= now;
    at += now;
  }
}

// A wavefront per row: rows of a few hundred states.
constexpr int kRowsPerGroup = 4;
__global__ void __launch_bounds__(64 * kRowsPerGroup) k_label_rows(LabelArgs a) {
  extern __shared__ uint32_t lds[];
  __shared__ uint2 deals[kRowsPerGroup][64];
  const uint32_t wave = wave_id(), lane = lane_id();
  const int64_t n = (int64_t)blockIdx.x * kRowsPerGroup + wave;
  if (n >= a.N) return;
  uint32_t* bits = lds + wave * a.words;
  const int64_t i0 = max(a.row[n], (int64_t)0), i1 = min(a.row[n + 1], a.n_states);
  for (uint32_t i = lane; i < a.words; i += 64) bits[i] = 0;
  __builtin_amdgcn_wave_barrier();
  for (int64_t i = i0; i < i1; i += 64)
    add_labels(a, i + lane < i1 ? (uint32_t)a.states[i + lane] : a.S, bits, deals[wave]);
  uint32_t* out = a.mask + n * a.ld;
  for (uint32_t i = lane; i < a.words; i += 64) out[i] = bits[i];
}

// `parts` workgroups per row.  With LDS the row's bits are gathered there and, of
// several workgroups, joined in memory; without, set in memory (k_label_zero has
// emptied it in both cases).
template <bool LDS>
__global__ void __launch_bounds__(1024) k_label_sets(LabelArgs a) {
  extern __shared__ uint32_t lds[];
  __shared__ uint2 deals[16][64];
  const uint32_t wave = wave_id(), lane = lane_id();
  const int64_t n = blockIdx.x / a.parts;
  const uint32_t part = blockIdx.x % a.parts;
  uint32_t* out = a.mask + n * a.ld;
  uint32_t* bits = LDS ? lds : out;
  const int64_t r0 = max(a.row[n], (int64_t)0), r1 = min(a.row[n + 1], a.n_states), len = max(r1 - r0, (int64_t)0);
  const int64_t i0 = r0 + len * part / a.parts, i1 = r0 + len * (part + 1) / a.parts;
  if (LDS) {
    for (uint32_t i = threadIdx.x; i < a.words; i += 1024) bits[i] = 0;
    __syncthreads();
  }
  for (int64_t i = i0 + wave * 64; i < i1; i += 1024)
    add_labels(a, i + lane < i1 ? (uint32_t)a.states[i + lane] : a.S, bits, deals[wave]);
  if (!LDS) return;
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < a.words; i += 1024) {
    if (a.parts == 1)
      out[i] = bits[i];
    else if (bits[i])
      atomicOr(&out[i], bits[i]);
  }
}

__global__ void __launch_bounds__(256) k_label_zero(LabelArgs a) {
  const uint64_t all = (uint64_t)a.N * a.words;
  for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256)
    a.mask[(int64_t)(i / a.words) * a.ld + (int64_t)(i % a.words)] = 0;
}

}  // namespace wd

using namespace wd;

extern "C" wd_status wd_label_masks(const wd_graph* g, int64_t N, const int64_t* off, const int32_t* states,
                                    int64_t n_states, uint32_t* mask, int64_t mask_ld, void* stream) {
  if (!g) return fail(WD_EINVAL, "label_masks: null graph");
  if (N < 0 || n_states < 0) return fail(WD_EINVAL, "label_masks: negative count");
  const uint32_t words = (g->P + 31) / 32;
  if (mask_ld < (int64_t)words) return fail(WD_EINVAL, "label_masks: mask_ld below ceil(num_pdfs / 32)");
  if (N == 0) return WD_OK;
  if (!off || !mask || (n_states && !states)) return fail(WD_EINVAL, "label_masks: null array");
  if ((uintptr_t)off & 7 || (uintptr_t)states & 3 || (uintptr_t)mask & 3)
    return fail(WD_EINVAL, "label_masks: misaligned array");
  if (N > INT32_MAX / 64) return fail(WD_EINVAL, "label_masks: too many rows for one call");
  LabelArgs a{g->dg.off, g->dg.ilabel_id, g->dg.S, words, 1, g->A, N, n_states, mask_ld, off, states, mask};
  hipStream_t s = (hipStream_t)stream;
  // The rows' own lengths are on the device: the average decides (one long set among
  // short ones is walked by one wavefront).  Of 500000 states: 4000 sets of 300 states 28
  // us a wavefront each and 38 a workgroup each, of 1200 82 and 92.  Few sets would
  // be faster by workgroups below the bound already: 300 of 300 states 14 and 9.
  const int64_t mean = n_states / N;
  constexpr uint32_t kRowWords = 3584, kLdsWords = 12288;  // (64 KB of LDS, the deals among it)
  if (mean <= 512 && words <= kRowWords) {
    hipLaunchKernelGGL(k_label_rows, dim3((uint32_t)((N + kRowsPerGroup - 1) / kRowsPerGroup)), dim3(64 * kRowsPerGroup),
                       kRowsPerGroup * words * 4, s, a);
    return hip_check(hipGetLastError(), "label_masks");
  }
  // long rows, few of them: several workgroups each, of 4096 states or more (30 sets of
  // 20000 states 32 us, 85 with one workgroup a set, 27 with parts of 1024; 300 sets 82, 143
  // and 82)
  a.parts = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(mean / 4096, (1023 + N) / N));
  if (a.parts > 1 || words > kLdsWords) {
    const uint64_t all = (uint64_t)N * words;
    hipLaunchKernelGGL(k_label_zero, dim3((uint32_t)std::min<uint64_t>((all + 255) / 256, 4096)), dim3(256), 0, s, a);
  }
  // (a launch has fewer than 2^32 threads: more rows than that take several)
  const int64_t most = ((1 << 22) - 1) / a.parts;
  for (; a.N > 0; a.N -= most, a.row += most, a.mask += most * mask_ld) {
    const dim3 grid((uint32_t)(std::min(most, a.N) * a.parts));
    if (words <= kLdsWords)
      hipLaunchKernelGGL(k_label_sets<true>, grid, dim3(1024), words * 4, s, a);
    else
      hipLaunchKernelGGL(k_label_sets<false>, grid, dim3(1024), 0, s, a);
  }
  return hip_check(hipGetLastError(), "label_masks");
}
