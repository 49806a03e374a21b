// What the sources of the C ABI share: errors, the checks of a model and a batch, uploads.
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

#include "../../include/wisp.h"

namespace wisp {

// keeps the message for wisp_last_error and returns st
wisp_status fail(wisp_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
wisp_status check_model(const wisp_model *m, bool need_weights);
// forward: the call runs the model, so prompt rows count towards the batch's rows
wisp_status check_desc(const wisp_batch_desc *d, bool need_pages, bool forward);
// the error of the launches since the last check
wisp_status hip_check(const char *what);
// compute units of the current device (attention work lists are sized to them)
int device_cus();
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
// host integers to device memory in stream order: through pinned staging, or as kernel arguments
// (a few KB per launch), which a stream that is being captured needs
wisp_status upload_ints(const std::vector<int32_t> &host, void *dst, hipStream_t s);
wisp_status upload_ints_by_arguments(const std::vector<int32_t> &host, void *dst, hipStream_t s);

}  // namespace wisp
