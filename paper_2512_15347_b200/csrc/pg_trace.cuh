// Named ranges around library calls for timeline tools.
#pragma once

#include <nvtx3/nvToolsExt.h>

namespace pg {

// A range as long as the call (NVTX; a no-op costing a pointer test when no tool is attached).
struct TraceRange {
  explicit TraceRange(const char* name) { nvtxRangePushA(name); }
  ~TraceRange() { nvtxRangePop(); }
  TraceRange(const TraceRange&) = delete;
  TraceRange& operator=(const TraceRange&) = delete;
};

}  // namespace pg
