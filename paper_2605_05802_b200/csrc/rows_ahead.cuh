// Rows that a kernel copies ahead (see adjust.cu).  Plain C++ as well, so that the last sizes can be checked on the host.
#pragma once

#ifdef __CUDACC__
#define SR_ROWS __host__ __device__ __forceinline__
#else
#define SR_ROWS static inline
#endif

namespace sr {

// Whether there is a row `by` behind `row` before `end`, for end >= 1 and 0 <= by < 2^31.  A call may have 2^31 - 1 rows: the row's own number is
// not worked out, it may need 32 bits and a sign.
SR_ROWS bool row_ahead(int row, int by, int end) { return row < end - by; }

}  // namespace sr
