// fe_host.h -- what the files with C entry points share: errors, argument checks
// and profiler ranges.  Not part of the public ABI.
#pragma once

#include <rocprofiler-sdk-roctx/roctx.h>

#include "../../include/fe.h"
#include "fe_internal.h"

namespace fe {

// Formats the calling thread's fe_last_error message and returns st.
fe_status fail(fe_status st, const char *fmt, ...);

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

#define FE_TRY(x)                                                           \
  do {                                                                      \
    hipError_t e_ = (x);                                                    \
    if (e_ != hipSuccess) return fail(FE_E_HIP, "%s: %s", #x, hipGetErrorString(e_)); \
  } while (0)

// A roctx range over a host scope: the entry points, the pass and its layers
// show up by name on a rocprofv3 --marker-trace timeline (host time: when the
// work was enqueued, or captured).
struct Range {
  explicit Range(const char *name) { roctxRangePushA(name); }
  ~Range() { roctxRangePop(); }
  Range(const Range &) = delete;
  Range &operator=(const Range &) = delete;
};

}  // namespace fe
