// C-ABI entry point of attention with a sliding window.
#include "as_attend_host.cuh"

namespace asx {

ASX_BOUNDS_READER(bounds_window)

}  // namespace asx

using namespace asx;

extern "C" {

int as_cache4_attend_window(const as_cache4* cache, const void* d_q, long long q_ld, int dtype, int lanes, int T, int q_heads,
                            const int32_t* d_table, int max_pages, const int32_t* d_len, double scale, int N, const int32_t* d_shared,
                            int window, int sinks, void* d_out, float* d_lse, int32_t* d_lane_status, void* d_work, size_t work_bytes,
                            void* stream) {
    if (window < 1 || sinks < 0) return set_err(AS_ERR_INVALID_ARG, "window = %d must be >= 1, sinks = %d >= 0", window, sinks);
    // (a lane has at most 2^30 positions)
    constexpr int most = 1 << 30;
    return attend<true>(cache, d_q, q_ld, dtype, lanes, T, q_heads, d_table, max_pages, d_len, scale, N, d_shared, window < most ? window : most,
                        sinks < most ? sinks : most, d_out, d_lse, d_lane_status, d_work, work_bytes, stream);
}

}  // extern "C"
