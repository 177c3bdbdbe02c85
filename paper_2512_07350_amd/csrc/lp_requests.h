// The rows of several requests packed one after the other (lp_requests), as kernels take them (not installed).
#pragma once
#include <stdint.h>

#include "lp.h"

namespace lp {

// Request r owns rows start[r] .. start[r + 1] - 1; entries past the last request lie behind every row, so that a lane
// of a wavefront can look at each of them.
struct RequestTable {
    int32_t count;
    int32_t start[LP_MAX_REQUESTS + 1];
    int64_t rows() const { return count > 0 ? start[count] : 0; }
};

inline int make_request_table(const lp_requests *q, RequestTable *out) {
    if (q == nullptr || q->count < 0) return LP_ERR_INVALID_ARG;
    if (q->count > LP_MAX_REQUESTS) return LP_ERR_LIMIT;
    if (q->count > 0 && (q->start == nullptr || q->start[0] != 0)) return LP_ERR_INVALID_ARG;
    for (int r = 0; r < q->count; ++r)
        if (q->start[r + 1] < q->start[r]) return LP_ERR_INVALID_ARG;
    if (q->count > 0 && q->start[q->count] >= INT32_MAX) return LP_ERR_UNSUPPORTED;
    out->count = q->count;
    for (int r = 0; r <= LP_MAX_REQUESTS; ++r) out->start[r] = r <= q->count && q->count > 0 ? int32_t(q->start[r]) : INT32_MAX;
    return LP_OK;
}

#ifdef __HIPCC__
// The request of row `row`, for all 64 lanes of a wavefront; ends is start[lane + 1].
__device__ __forceinline__ int request_of(int32_t ends, int32_t row) { return __popcll(__ballot(ends <= row)); }
#endif

}  // namespace lp
