// How a group of threads goes over rows in the norms' kernels.  Plain C++, for the device and the host.
#pragma once

#ifdef __CUDACC__
#define VARDROP_WALK_FN __host__ __device__ __forceinline__
#else
#define VARDROP_WALK_FN inline
#endif

namespace vardrop {

// A call has fewer than 2^31 rows, and a walk looks up to three steps behind the last one (of 9472 rows, where rows are narrow): past what an int holds.
typedef unsigned RowIndex;

struct RowSteps {
    RowIndex n, step;
    VARDROP_WALK_FN bool there(RowIndex i) const { return i < n; }
    VARDROP_WALK_FN bool goes_on(RowIndex i, RowIndex behind) const { return i < n + behind; }
};

}  // namespace vardrop
