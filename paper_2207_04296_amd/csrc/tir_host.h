// What the entry points of the other translation units share with tir_api.hip: error reports and the workspace a caller registered.
#pragma once
#include <hip/hip_runtime.h>
#include "tir.h"

namespace tir {

// Records the message for tir_last_error and returns st.
tir_status host_error(tir_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// The workspace registered for `stream` of the current device (tir_set_workspace): partial sums and zeroed arrival counters.  partial is
// null where there is none: what needs it runs unsplit then.
struct StreamWorkspace {
    void* partial;
    unsigned* count;
    int64_t bytes, counters;
};
StreamWorkspace stream_workspace(hipStream_t stream);

inline bool host_aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace tir
