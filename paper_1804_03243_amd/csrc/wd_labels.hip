// Label masks from the decoding graph: for every row, the input labels that
// leave a set of states, as bits.
//
//   mask[n] = OR over s in states(n), over arcs a of s with ilabel k >= 1, of bit k - 1
//
// The caller's arcs of a state are a run of the label array (by caller arc
// id), which starts at the number of emitting plus epsilon arcs before it, so
// an arc costs a 4-byte read.
#include <algorithm>

#include "wd_host.h"
#include "wd_num.h"

namespace wd {

// A row's words in LDS up to this many; longer ones straight in memory.
constexpr uint32_t kLabelWords = 16384;

struct LabelArgs {
  const uint4* off;
  const int32_t* ilabel;
  uint32_t S, words;
  int64_t N, n_states, ld;
  const int64_t* row;
  const int32_t* states;
  uint32_t* mask;
};

// One workgroup per row.
template <bool LDS>
__global__ void __launch_bounds__(256) k_label_masks(LabelArgs a) {
  extern __shared__ uint32_t bits[];
  for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
    uint32_t* out = a.mask + n * a.ld;
    uint32_t* w = LDS ? bits : out;
    for (uint32_t i = threadIdx.x; i < a.words; i += 256) w[i] = 0;
    __syncthreads();
    const int64_t i0 = max(a.row[n], (int64_t)0), i1 = min(a.row[n + 1], a.n_states);
    for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
      const uint32_t s = (uint32_t)a.states[i];
      if (s >= a.S) continue;
      const uint4 o = a.off[s], e = a.off[s + 1];
      for (uint32_t k = o.x + o.y; k < e.x + e.y; ++k) {
        const uint32_t l = (uint32_t)a.ilabel[k] - 1u;
        if (l < a.words * 32u) atomicOr(&w[l >> 5], 1u << (l & 31));
      }
    }
    if (LDS) {
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < a.words; i += 256) out[i] = bits[i];
    }
    __syncthreads();
  }
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
  LabelArgs a{g->dg.off, g->dg.ilabel_id, g->dg.S, words, N, n_states, mask_ld, off, states, mask};
  const uint32_t grid = (uint32_t)std::min<int64_t>(N, 1 << 20);
  hipStream_t s = (hipStream_t)stream;
  if (words <= kLabelWords)
    hipLaunchKernelGGL(k_label_masks<true>, dim3(grid), dim3(256), words * 4, s, a);
  else
    hipLaunchKernelGGL(k_label_masks<false>, dim3(grid), dim3(256), 0, s, a);
  return hip_check(hipGetLastError(), "label_masks");
}
