// What the host sides of the C ABI share (api.cu, serve_api.cu): refusing an argument, and the
// profiler range of a call.
#pragma once

#ifndef MPQ_NO_NVTX
#include <nvtx3/nvToolsExt.h>
#endif

#include "mpq_internal.cuh"

// One NVTX range per C-ABI call (named after the entry point), so that a profiler's timeline shows
// which call enqueued which kernels; with no tool attached a range costs a few nanoseconds.
// Build with -DMPQ_NO_NVTX to leave them out.
namespace {
struct CallRange {
#ifndef MPQ_NO_NVTX
    explicit CallRange(const char *name) { nvtxRangePushA(name); }
    ~CallRange() { nvtxRangePop(); }
#else
    explicit CallRange(const char *) {}
#endif
};
}  // namespace

#define REQUIRE(cond, status, ...)       \
    do {                                 \
        if (!(cond)) {                   \
            mpq::set_error(__VA_ARGS__); \
            return (status);             \
        }                                \
    } while (0)
