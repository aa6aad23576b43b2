// What a decode's status says, apart from the kernels that set it so that it can be
// checked on the host.
#pragma once

#include <stdint.h>

#include "../../include/wfstdec.h"

namespace wd {

// LaneInfo::status: a wd_status in the low byte; for an internal consistency failure
// caught by a kernel's own checks (WD_EDEVICE) the check above it.
constexpr int32_t kStatusInternal = WD_EDEVICE;
constexpr int32_t internal_status(int32_t check) { return kStatusInternal | check << 8; }
constexpr int32_t kClusterWait = internal_status(1);
constexpr int32_t kKeptCount = internal_status(2);
constexpr int32_t kWarmPayload = internal_status(3);
constexpr int32_t kGridFrame = internal_status(4);
constexpr int32_t kSweepWait = internal_status(5);
constexpr int32_t kLinkTarget = internal_status(6);
constexpr int32_t kTraceback = internal_status(7);

inline wd_status status_of(int32_t s) { return (wd_status)(s & 0xff); }

inline const char* status_message(int32_t s) {
#define WD_INTERNAL "decode: a kernel's internal consistency check failed: "
  switch (s) {
    case WD_ENOPATH: return "decode: no token survived a frame";
    case WD_EINVAL: return "decode: log-likelihoods contain NaN, +inf or values above 1e30";
    case WD_ECAPACITY: return "decode: workspace capacity exceeded; see stats.needed";
    case kClusterWait: return WD_INTERNAL "a workgroup waited too long for the others of a large frame";
    case kKeptCount: return WD_INTERNAL "a frame's kept tokens were counted twice with different results";
    case kWarmPayload: return WD_INTERNAL "a weight or log-likelihood of a payload that none has";
    case kGridFrame: return WD_INTERNAL "a chip-wide frame's tokens or links do not match their counts";
    case kSweepWait: return WD_INTERNAL "a workgroup waited too long for the others of the pruning sweep";
    case kLinkTarget: return WD_INTERNAL "a lattice link's destination is not among its frame's tokens";
    case kTraceback: return WD_INTERNAL "the best path met an inconsistent predecessor";
  }
  return status_of(s) == WD_EDEVICE ? "decode: a kernel's internal consistency check failed" : "decode failed";
#undef WD_INTERNAL
}

}  // namespace wd
