// crf_plan.h -- the plan object and the status helpers that the C entry points share.
//
// Not part of the public ABI (that is include/crf_inside.h).
#pragma once

#include <vector>

#include "crf_internal.h"

struct crf_plan {
    int device = -1;
    int32_t B = 0, n1 = 0, L = 1, max_len = 0;
    uint32_t flags = 0;
    std::vector<void *> allocations;
    crf::KernelPlan kp{};
    int64_t ws_bytes = 0;          // device workspace owned
    int64_t scratch_bytes = 0;     // of it, what the no-allocation call needs at least
    int32_t split_ws_count = 0;    // sentences with CKY split tables in the workspace
    int32_t workspace_users = 0;   // sentences using the workspace in some call
    int64_t cells = 0;             // squares of the lengths, summed (see KernelPlan::post_cells)
};

namespace crf {

// Set the calling thread's last error and return its status.
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int ok();
int hip_fail(hipError_t e, const char *where);
// CRF_OK when the plan's device is the current one.
int check_device(const crf_plan *plan);

}  // namespace crf
