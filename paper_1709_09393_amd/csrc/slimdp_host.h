// What the host sides of the library's translation units share: the few fields of a context that the training operators need,
// and its error message.  The context itself stays private to slimdp.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "slimdp.h"

#define SLIMDP_HIDDEN __attribute__((visibility("hidden")))

namespace slimdp {

struct HostView {
    uint32_t max_workers;
    int device;
    hipStream_t stream;
    uint32_t* status;          // device word that slimdp_synchronize reports
};
SLIMDP_HIDDEN HostView host_view(const slimdp_ctx* ctx);
SLIMDP_HIDDEN int host_fail(slimdp_ctx* ctx, int code, const char* fmt, ...) __attribute__((format(printf, 3, 4)));

// Status bits of kernels (see slimdp_synchronize): 1 and 2 belong to the explorer's lists.
constexpr uint32_t STATUS_TEACHER = 4u;          // a teacher's index lies outside the vocabulary

}  // namespace slimdp
