// entry.cuh -- what the C entry points share: the error message and status of
// the calling thread, the checks of pointers, and the host-side fault injection.
#pragma once
#include <stdint.h>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "rdn.h"

namespace rdn {
// Records the thread's message (rdn_last_error) and returns st.
rdn_status_t entry_fail(rdn_status_t st, const char *fmt, ...);
// Clears the message; RDN_OK.
rdn_status_t entry_ok();
// The failures RDN_FAULT_INJECT asks for, after validation; else RDN_OK.
rdn_status_t entry_injected(const char *fn);
// The outcome of the launches.
rdn_status_t entry_cuda(const char *fn, cudaError_t e);

// An NVTX range named after the entry point for the duration of the call
// (host side: validation and enqueueing), seen by profilers and free without one.
struct CallRange {
  explicit CallRange(const char *fn) { nvtxRangePushA(fn); }
  ~CallRange() { nvtxRangePop(); }
};
}  // namespace rdn
