// Named ranges around the public calls for timeline tools (NVTX; compiled in with -DTD_NVTX, the
// header-only nvtx3 that ships with the toolkit; otherwise the macro is empty).
#pragma once
#ifdef TD_NVTX
#include <nvtx3/nvToolsExt.h>
namespace {
struct TdRange {
    explicit TdRange(const char *name) { nvtxRangePushA(name); }
    ~TdRange() { nvtxRangePop(); }
};
}  // namespace
#define TD_RANGE(name) TdRange td_range_guard(name)
#else
#define TD_RANGE(name) do { } while (0)
#endif
