// Checked builds (-DAS_BOUNDS_CHECK): every index into a ring stage, a hit or candidate list, a
// rank array, a histogram, a chunk array, the mass table or a row buffer goes through ASX_AT; of the cache,
// attention and page kernels the places in tiles, tables, rings, shared matrices, TMEM columns, joins, states
// in scratch, query and output rows, page lists and page numbers that were computed.  An
// index outside [0, n) is recorded (the count of failures and the first one's site, index and
// bound) and replaced by 0, so that the access stays in bounds: nothing traps, and the host reads
// the record after the launch.  In ordinary builds ASX_AT(i, n, site) is just i.
#pragma once
#include <cuda_runtime.h>

namespace asx {

#ifdef AS_BOUNDS_CHECK
static __device__ int g_asx_bounds[4];
__device__ __forceinline__ bool asx_in(long long i, long long n, int site) {
    if (i >= 0 && i < n) return true;
    if (atomicAdd(&g_asx_bounds[0], 1) == 0) {
        g_asx_bounds[1] = site;
        g_asx_bounds[2] = (int)i;
        g_asx_bounds[3] = (int)n;
    }
    return false;
}
#define ASX_AT(i, n, site) (asx_in((long long)(i), (long long)(n), (site)) ? (i) : 0)
// defines a translation unit's function that copies its record out and resets it
#define ASX_BOUNDS_READER(name)                                                                          \
    int name(int* h_out4, int reset) {                                                                   \
        int zero[4] = {0, 0, 0, 0};                                                                      \
        if (h_out4 && cudaMemcpyFromSymbol(h_out4, g_asx_bounds, sizeof(zero)) != cudaSuccess) return -3; \
        if (reset && cudaMemcpyToSymbol(g_asx_bounds, zero, sizeof(zero)) != cudaSuccess) return -3;      \
        return 0;                                                                                        \
    }
#else
#define ASX_AT(i, n, site) (i)
#define ASX_BOUNDS_READER(name)
#endif

}  // namespace asx
