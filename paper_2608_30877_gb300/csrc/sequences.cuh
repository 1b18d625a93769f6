// Sequences of a packed batch: rows [seq_start[s], seq_start[s + 1]) of a table [nseq + 1].
#pragma once

#include <cuda_runtime.h>
#include <cstdint>

#include "ptx.cuh"

namespace w4a16 {

// The sequence of row m with its rows, -1 outside every sequence.
__device__ __forceinline__ int sequence_of(const int32_t* seq_start, int nseq, int m, int* begin, int* end) {
    int lo = 0, hi = nseq;  // the last sequence that starts at m or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (seq_start[mid] <= m) lo = mid; else hi = mid - 1;
    }
    if (lo >= nseq) return -1;
    *begin = seq_start[lo];
    *end = seq_start[lo + 1];
    return *begin <= m && m < *end ? lo : -1;
}

// Records a table that decreases or leaves [0, M], also where no row shows it.  Called by every thread
// of the CTAs of gridDim.x.
__device__ __forceinline__ void check_starts(const int32_t* seq_start, int nseq, int M, int* status) {
    for (int64_t s = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; s < nseq;
         s += static_cast<int64_t>(gridDim.x) * blockDim.x)
        if (seq_start[s] > seq_start[s + 1] || seq_start[s] < 0 || seq_start[s + 1] > M)
            record_status(status, 1 /* W4A16_ERR_INVALID_ARG */);
}

}  // namespace w4a16
